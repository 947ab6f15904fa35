"""Operators over a paged cache of request histories, as measurable cases.

A request's keys and values live in pages between its visits: K, V [layers, n_pages, page, H_kv, dh], a table of page
ids per slot, a length per slot, a number of holders per page.  Kinds of case:

  attend   attention of every request's new rows over its slot of the cache: one event (decode), a chunk of new events or
           a whole history (causal), or the candidates of the request (all keys visible)
  step     a serving step's bookkeeping: last step's forks are given back, slots are forked from their parents, grown by a
           chunk (a shared last page is copied first) and the chunk's keys and values written, for all layers
  compact  pages in use are moved below a line, tables and holders follow

Lengths, counts and which slot is whose belong to the case ("segments"), page ids and values to the seed.
"""
import math
import random

import numpy as np
import torch

own = False

BF16, F32 = "bf16", "f32"
_DTYPE = {BF16: torch.bfloat16, F32: torch.float32}
_SIZE = {BF16: 2, F32: 4}

_ATTEND = {"kind": "attend", "dtype": BF16, "causal": True, "cap": 0.0, "bias": False, "doc": 0, "prefix": 0.0}


def listed():
    return [
        # The smallest call: one new event of each of four users with short histories; launches are the time.
        dict(_ATTEND, name="event_small", R=4, n_lo=1, n_hi=1, len_lo=60, len_hi=900, Hkv=8, G=1, dh=64, page=16, segments=1),
        # One new event of a batch of users, grouped heads: what a decoding loop does at every step.
        dict(_ATTEND, name="event_batch", R=64, n_lo=1, n_hi=1, len_lo=500, len_hi=8000, Hkv=8, G=4, dh=128, page=64, segments=2),
        # A few users whose histories are very long, one to three events each, scores that fall with distance.
        dict(_ATTEND, name="event_long", R=3, n_lo=1, n_hi=3, len_lo=60000, len_hi=180000, Hkv=4, G=8, dh=128, page=128, bias=True,
             segments=3),
        # Sessions of new events over the histories of the ranking workload: 8 heads of 64, up to 2048 keys.
        dict(_ATTEND, name="session_chunk", R=24, n_lo=8, n_hi=120, len_lo=200, len_hi=2048, Hkv=8, G=1, dh=64, page=16, segments=4),
        # First visits: whole histories at once, capped scores, sessions that do not see one another, a visible prefix.
        dict(_ATTEND, name="first_visits", R=6, n_lo=1100, n_hi=2900, len_lo=1, len_hi=1, Hkv=4, G=4, dh=128, page=32, cap=30.0,
             doc=700, prefix=0.2, segments=5),
        # The heaviest call: a long chunk over a longer history.
        dict(_ATTEND, name="long_chunk", R=1, n_lo=2048, n_hi=2048, len_lo=16401, len_hi=16401, Hkv=8, G=4, dh=128, page=128, segments=6),
        # Candidates over the cached histories: ranking, 8 heads of 64, 2048 keys.
        dict(_ATTEND, name="candidates", R=32, n_lo=200, n_hi=1000, len_lo=1700, len_hi=2048, Hkv=8, G=1, dh=64, page=64, causal=False,
             segments=7),
        # fp32 storage, for callers that do not round to bf16: short histories, small pages.
        dict(_ATTEND, name="chunk_f32", dtype=F32, R=6, n_lo=1, n_hi=60, len_lo=30, len_hi=600, Hkv=4, G=2, dh=64, page=8, segments=8),
        # A small step: four users forked once each, a few events, two layers.
        {"kind": "step", "name": "step_small", "dtype": BF16, "R": 4, "parents": 4, "layers": 2, "n_lo": 1, "n_hi": 5, "len_lo": 60,
         "len_hi": 500, "Hkv": 8, "dh": 64, "page": 16, "segments": 9},
        # A large one: 128 forks of 32 users, chunks of up to 200 events, eight layers.
        {"kind": "step", "name": "step_large", "dtype": BF16, "R": 128, "parents": 32, "layers": 8, "n_lo": 20, "n_hi": 200,
         "len_lo": 200, "len_hi": 4000, "Hkv": 8, "dh": 64, "page": 64, "segments": 10},
        # A small pool with holes.
        {"kind": "compact", "name": "compact_small", "dtype": BF16, "R": 8, "layers": 1, "len_lo": 20, "len_hi": 400, "Hkv": 4, "dh": 64,
         "page": 16, "fill": 0.5, "segments": 11},
        # A pool of thousands of pages and several layers, two thirds in use.
        {"kind": "compact", "name": "compact_large", "dtype": BF16, "R": 96, "layers": 6, "len_lo": 500, "len_hi": 4000, "Hkv": 8, "dh": 64,
         "page": 32, "fill": 0.65, "segments": 12},
    ]


def draw(rng):
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    segments = rng.randrange(100, 1 << 20)
    kind = rng.choice(["attend"] * 5 + ["step", "compact"])
    page = rng.choice([8, 16, 16, 24, 32, 64, 64, 128])
    if kind == "step":
        R = log_int(1, 128)
        n = log_int(1, 200)
        return {"kind": kind, "dtype": rng.choice([BF16, BF16, F32]), "R": R, "parents": log_int(1, R), "layers": rng.randint(1, 6),
                "n_lo": max(1, n // 4), "n_hi": n, "len_lo": log_int(1, 100), "len_hi": log_int(101, 3000),
                "Hkv": rng.choice([1, 2, 4, 8]), "dh": rng.choice([32, 64, 64, 128 if n < 100 else 64]), "page": page,
                "segments": segments}
    if kind == "compact":
        return {"kind": kind, "dtype": rng.choice([BF16, BF16, F32]), "R": log_int(1, 100), "layers": rng.randint(1, 4),
                "len_lo": log_int(1, 100), "len_hi": log_int(101, 2500), "Hkv": rng.choice([1, 2, 4, 8]),
                "dh": rng.choice([32, 64, 64, 128]), "page": page, "fill": round(rng.uniform(0.3, 0.95), 2), "segments": segments}
    case = dict(_ATTEND, segments=segments, page=page)
    mode = rng.choice(["event", "event", "chunk", "chunk", "visit", "candidates", "f32"])
    Hkv, G, dh = rng.choice([1, 2, 4, 8]), rng.choice([1, 1, 2, 3, 4, 5, 8]), rng.choice([32, 64, 64, 128, 128])
    if mode == "f32":
        case["dtype"] = F32
        Hkv, G, dh = rng.choice([1, 2, 4]), rng.choice([1, 2, 3]), rng.choice([32, 64])
    H = Hkv * G
    if mode == "event":
        hi = log_int(30, 60000)
        R = log_int(1, max(1, min(256, 400_000_000 // (hi * Hkv * dh * 2))))
        n = rng.choice([1, 1, 1, 2, 4])
    elif mode == "f32":
        hi, R, n = log_int(20, 600), log_int(1, 12), log_int(1, 64)
    else:
        hi = log_int(200, 8000)
        n = hi if mode == "visit" else log_int(8, 1000)
        hi = min(hi, 3500) if mode == "visit" else hi
        n = min(n, hi)
        R = log_int(1, max(1, min(64, 400_000_000 // (hi * n * H))))
    case.update(R=R, n_lo=max(1, n // 3), n_hi=n, len_lo=max(1, hi // 8), len_hi=hi, Hkv=Hkv, G=G, dh=dh)
    if mode == "visit":
        case.update(n_lo=max(1, n // 2), len_lo=1, len_hi=1)
    if mode == "candidates":
        case["causal"] = False
    else:
        case.update(cap=rng.choice([0.0, 0.0, 0.0, 20.0, 50.0]), doc=rng.choice([0, 0, 0, log_int(20, 2000)]),
                    prefix=rng.choice([0.0, 0.0, 0.3]) if mode in ("chunk", "visit") else 0.0)
    case["bias"] = rng.random() < 0.3
    return case


# ---------------------------------------------------------------------------------- sizes, from the case alone
def _log_ints(rng, lo, hi, n):
    return [min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))) for _ in range(n)]


def _sizes(case):
    """New rows and cached positions of each request, on the host; what else the kinds need."""
    rng = random.Random(case["segments"])
    R, page = case["R"], case["page"]
    z = {}
    if case["kind"] == "attend":
        n = _log_ints(rng, case["n_lo"], case["n_hi"], R)
        L = _log_ints(rng, case["len_lo"], case["len_hi"], R)
        z["n"] = n
        z["len"] = [max(a, b) for a, b in zip(n, L)] if case["causal"] else L
        z["doc"] = [max(1, int(case["doc"] * rng.uniform(0.5, 1.5))) if case["doc"] else 0 for _ in range(R)]
        z["prefix"] = [int(case["prefix"] * l * rng.uniform(0.5, 1.5)) for l in z["len"]]
        z["slots"] = R + 3
        z["held"] = z["len"]
    elif case["kind"] == "step":
        z["n"] = _log_ints(rng, case["n_lo"], case["n_hi"], R)
        z["held"] = _log_ints(rng, case["len_lo"], case["len_hi"], case["parents"])
        z["parent"] = [rng.randrange(case["parents"]) for _ in range(R)]
        z["slots"] = case["parents"] + R
        z["grown"] = sum(-(-(z["held"][p] + n) // page) - -(-z["held"][p] // page) + (1 if z["held"][p] % page else 0)
                         for p, n in zip(z["parent"], z["n"]))
    else:
        z["held"] = _log_ints(rng, case["len_lo"], case["len_hi"], R)
        z["slots"] = R
    z["used"] = sum(-(-l // page) for l in z["held"])
    if case["kind"] == "attend":
        z["n_pages"] = z["used"] + 1 + z["used"] // 16
    elif case["kind"] == "step":
        z["n_pages"] = z["used"] + z["grown"] + 2 + z["used"] // 8
    else:
        z["n_pages"] = max(z["used"] + 1, int(z["used"] / case["fill"]))
    z["width"] = -(-(max(z["held"]) + max(z.get("n", [0]))) // page) + 1
    return z


# ---------------------------------------------------------------------------------- inputs
def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    z = _sizes(case)
    dtype, page, Hkv, dh = _DTYPE[case["dtype"]], case["page"], case["Hkv"], case["dh"]

    def normal(*shape, std=1.0):
        return (torch.randn(shape, generator=g, device="cuda", dtype=torch.float32 if case["dtype"] == F32 else dtype) * std).to(dtype)

    def ints(v):
        return torch.tensor(v, dtype=torch.int32, device="cuda")

    s = {"case": case, "z": z}
    shape = (case.get("layers", 1), z["n_pages"], page, Hkv, dh)
    s["K"], s["V"] = normal(*shape), normal(*shape)
    # which slots hold something, and where: slots in an order of the case's, pages in one of the seed's
    order = list(range(z["slots"]))
    random.Random(case["segments"] + 1).shuffle(order)
    held = torch.tensor(z["held"], device="cuda")
    pages = (held + page - 1) // page
    first = torch.cumsum(pages, 0) - pages
    col = torch.arange(z["width"], device="cuda")
    ids = torch.randperm(z["n_pages"], generator=g, device="cuda")
    row = torch.where(col[None] < pages[:, None], ids[(first[:, None] + col[None]).clamp(max=z["n_pages"] - 1)], torch.full_like(col, -1)[None])
    slots = ints(order[:len(z["held"])])
    s["table"] = torch.full((z["slots"], z["width"]), -1, dtype=torch.int32, device="cuda")
    s["table"][slots.long()] = row.to(torch.int32)
    s["lens"] = torch.zeros(z["slots"], dtype=torch.int32, device="cuda")
    s["lens"][slots.long()] = held.to(torch.int32)
    s["refs"] = torch.zeros(z["n_pages"], dtype=torch.int32, device="cuda")
    s["refs"][ids[:z["used"]]] = 1
    s["report"] = torch.zeros(2, dtype=torch.int32, device="cuda")
    if "n" in z:
        off = np.concatenate([[0], np.cumsum(z["n"])]).astype(np.int32)
        s["offsets_host"] = torch.from_numpy(off)
        s["offsets"] = s["offsets_host"].cuda()
        s["req"] = torch.from_numpy(np.repeat(np.arange(case["R"]), z["n"])).cuda()
        s["t"] = torch.arange(int(off[-1]), device="cuda") - s["offsets"].long()[s["req"]]
        N = int(off[-1])
    if case["kind"] == "attend":
        H = Hkv * case["G"]
        s["slots"] = slots
        s["Q"] = normal(N, H, dh, std=1.5)
        s["out"] = torch.empty((N, H, dh), dtype=dtype, device="cuda")
        s["slopes"] = 2.0 ** (-8.0 * torch.arange(1, H + 1, device="cuda") / H) if case["bias"] else None
        s["begin"] = s["prefix"] = None
        if case["doc"]:
            pos = (held - torch.tensor(z["n"], device="cuda"))[s["req"]] + s["t"]
            doc = torch.tensor(z["doc"], device="cuda")[s["req"]]
            s["begin"] = (pos // doc * doc).to(torch.int32)
        if case["prefix"]:
            s["prefix"] = ints(z["prefix"])
    elif case["kind"] == "step":
        s["children"] = ints(order[len(z["held"]):])
        s["parents"] = slots[torch.tensor(z["parent"], device="cuda")].contiguous()
        s["K_new"], s["V_new"] = normal(case["layers"], N, Hkv, dh), normal(case["layers"], N, Hkv, dh)
        s["first"] = torch.zeros(case["R"], dtype=torch.int32, device="cuda")
    else:
        s["table_out"], s["refs_out"] = torch.empty_like(s["table"]), torch.empty_like(s["refs"])
    return s


# ---------------------------------------------------------------------------------- one pass
def run(s):
    kind = s["case"]["kind"]
    if own:
        return _run_own(s, kind)
    return {"attend": _attend, "step": _step, "compact": _compact}[kind](s)


def _run_own(s, kind):
    from paper_2607_27744_b200 import binding as rocs
    if "cache" not in s:  # what a program keeps: the handle of its cache, the plan of a batch's rows, a workspace
        s["cache"] = rocs.cache_create(s["K"], s["V"], s["table"], s["lens"], s["refs"])
        if "offsets" in s:
            s["plan"] = rocs.plan_create(s["offsets"], s["offsets_host"])
        need = (rocs.cache_attention_workspace(s["cache"], s["plan"], s["Q"].shape[1]) if kind == "attend" else
                rocs.cache_workspace(s["cache"], s["case"]["R"]))
        s["workspace"] = torch.empty(need, dtype=torch.uint8, device="cuda")
    cache, case, ws = s["cache"], s["case"], s["workspace"]
    if kind == "attend":
        return rocs.cache_attention(cache, s["plan"], s["Q"], slots=s["slots"], causal=case["causal"], cap=case["cap"], slopes=s["slopes"],
                                    begin=s["begin"], prefix=s["prefix"], out=s["out"], workspace=ws)
    if kind == "compact":
        rocs.cache_compact(cache, table_out=s["table_out"], refs_out=s["refs_out"], report=s["report"], workspace=ws)
        return {"table": s["table_out"], "refs": s["refs_out"], "K": s["K"], "V": s["V"], "report": s["report"]}
    rocs.cache_truncate(cache, s["children"], workspace=ws)
    rocs.cache_fork(cache, s["parents"], s["children"], workspace=ws)
    first = rocs.cache_extend(cache, s["plan"], slots=s["children"], report=s["report"], first=s["first"], workspace=ws)
    for layer in range(case["layers"]):
        rocs.cache_append(cache, s["plan"], first, s["K_new"][layer], s["V_new"][layer], slots=s["children"], layer=layer)
    return {"table": s["table"], "lens": s["lens"], "refs": s["refs"], "K": s["K"], "V": s["V"], "first": first, "report": s["report"]}


def _attend(s):
    case, z = s["case"], s["z"]
    page, Hkv, G, dh = case["page"], case["Hkv"], case["G"], case["dh"]
    R, n_max, L_max = case["R"], max(z["n"]), max(z["len"])
    slots = s["slots"].long()
    L = s["lens"][slots].long()
    n = (s["offsets"][1:] - s["offsets"][:-1]).long()
    j = torch.arange(-(-L_max // page) * page, device="cuda")
    ids = s["table"][slots][:, :-(-L_max // page)].clamp(min=0).long()
    there = (j[None] < L[:, None])[:, :, None, None]
    k = torch.where(there, s["K"][0][ids].reshape(R, -1, Hkv, dh).float(), 0.0)
    v = torch.where(there, s["V"][0][ids].reshape(R, -1, Hkv, dh).float(), 0.0)
    t = torch.arange(n_max, device="cuda")
    rows = (s["offsets"][:-1].long()[:, None] + t[None]).clamp(max=s["Q"].shape[0] - 1)
    q = s["Q"][rows].float().reshape(R, n_max, Hkv, G, dh).permute(0, 2, 3, 1, 4).reshape(R, Hkv, G * n_max, dh)
    x = torch.matmul(q, k.permute(0, 2, 3, 1)).view(R, Hkv, G, n_max, -1).mul_(dh ** -0.5)
    if case["cap"]:
        x.div_(case["cap"]).tanh_().mul_(case["cap"])
    pos = (L - n)[:, None] + t[None] if case["causal"] else L[:, None].expand(R, n_max)  # candidates stand behind the last key
    if s["slopes"] is not None:
        x -= s["slopes"].float().view(1, Hkv, G, 1, 1) * (pos[:, :, None] - j).abs()[:, None, None]
    hi = L[:, None].expand(R, n_max)
    if case["causal"]:
        hi = pos + 1
        if s["prefix"] is not None:
            hi = torch.maximum(hi, s["prefix"].long()[:, None])
        hi = torch.minimum(hi, L[:, None])
    seen = j < hi[:, :, None]
    if s["begin"] is not None:
        seen &= j >= s["begin"].long()[rows][:, :, None]
    x.masked_fill_(~seen[:, None, None], -math.inf)
    x -= x.amax(-1, keepdim=True).clamp(min=-3e38)
    x.exp_()
    total = x.sum(-1, keepdim=True)
    o = torch.matmul(x.view(R, Hkv, G * n_max, -1), v.permute(0, 2, 1, 3)).view(R, Hkv, G, n_max, dh)
    o = torch.where(total > 0, o / total, 0.0).permute(0, 3, 1, 2, 4).reshape(R, n_max, Hkv * G, dh)
    return o[s["req"], s["t"]].to(s["Q"].dtype)


def _step(s):
    page, table, lens, refs = s["case"]["page"], s["table"], s["lens"], s["refs"]
    child, parent = s["children"].long(), s["parents"].long()
    col = torch.arange(table.shape[1], device="cuda")
    one = torch.ones((), dtype=torch.int32, device="cuda")
    # last step's children give their pages back
    has = col[None] < ((lens[child] + page - 1) // page)[:, None]
    refs.index_put_((table[child][has].long(),), -one, accumulate=True)
    # fork: the parent's pages, held once more
    L = lens[parent]
    has = col[None] < ((L + page - 1) // page)[:, None]
    table[child] = torch.where(has, table[parent], table[child])
    refs.index_put_((table[child][has].long(),), one, accumulate=True)
    # extend: the lowest free pages in order of request and position; a shared last page is replaced by a copy
    n = s["offsets"][1:] - s["offsets"][:-1]
    last = table[child, (L // page).long()].clamp(min=0).long()
    copied = (L % page != 0) & (n > 0) & (refs[last] > 1)
    start = (L + page - 1) // page - copied.int()
    count = (L + n + page - 1) // page - start
    before = torch.cumsum(count, 0) - count
    free = torch.argsort((refs != 0).to(torch.int32), stable=True)
    mine = (col[None] >= start[:, None]) & (col[None] < (start + count)[:, None])
    rank = (before[:, None] + col[None] - start[:, None]).clamp(min=0, max=free.numel() - 1)
    taken = torch.where(mine, free[rank].to(torch.int32), table[child])
    refs.index_put_((last[copied],), -one, accumulate=True)
    refs.index_put_((taken[mine].long(),), one, accumulate=True)
    table[child] = taken
    to = taken.gather(1, (L // page).long()[:, None])[:, 0].long()[copied]
    s["K"][:, to] = s["K"][:, last[copied]]
    s["V"][:, to] = s["V"][:, last[copied]]
    lens[child] = L + n
    s["first"].copy_(L)
    s["report"].copy_(torch.stack([torch.zeros_like(one), count.sum().to(torch.int32)]))
    # append
    pos = (L[s["req"]] + s["t"]).long()
    at = table[child[s["req"]], pos // page].long()
    s["K"][:, at, pos % page] = s["K_new"]
    s["V"][:, at, pos % page] = s["V_new"]
    return {"table": table, "lens": lens, "refs": refs, "K": s["K"], "V": s["V"], "first": s["first"], "report": s["report"]}


def _compact(s):
    page, table, refs = s["case"]["page"], s["table"], s["refs"]
    ids = torch.arange(refs.numel(), device="cuda")
    live = refs > 0
    line = live.sum()
    src = ids[live & (ids >= line)]
    dst = ids[~live & (ids < line)]
    to = ids.clone()
    to[src] = dst
    col = torch.arange(table.shape[1], device="cuda")
    has = col[None] < ((s["lens"] + page - 1) // page)[:, None]
    s["table_out"].copy_(torch.where(has, to[table.clamp(min=0).long()].to(torch.int32), table))
    s["refs_out"].copy_(refs)
    s["refs_out"][dst] = refs[src]
    s["refs_out"][src] = 0
    s["K"][:, dst] = s["K"][:, src]
    s["V"][:, dst] = s["V"][:, src]
    s["report"].copy_(torch.stack([torch.zeros_like(line), line]))
    return {"table": s["table_out"], "refs": s["refs_out"], "K": s["K"], "V": s["V"], "report": s["report"]}


# ---------------------------------------------------------------------------------- what a pass needs
def _visible(case, z):
    """(visible pairs of row and key, keys that some row of the request sees), over all requests."""
    pairs, keys = 0, 0
    for n, L, doc, prefix in zip(z["n"], z["len"], z["doc"], z["prefix"]):
        pos = L - n + np.arange(n)
        hi = np.full(n, L)
        if case["causal"]:
            hi = np.minimum(np.maximum(pos + 1, prefix if case["prefix"] else 0), L)
        lo = pos // doc * doc if doc else np.zeros(n, int)
        pairs += int(np.maximum(hi - lo, 0).sum())
        keys += int(max(0, hi.max() - lo.min()))
    return pairs, keys


def work(case):
    z, e = _sizes(case), _SIZE[case["dtype"]]
    width = case["Hkv"] * case["dh"]
    if case["kind"] == "attend":
        pairs, keys = _visible(case, z)
        rows = sum(z["n"]) * width * case["G"]
        return {"bytes": 2 * rows * e + 2 * keys * width * e + 4 * (keys // case["page"] + 4 * case["R"]),
                "flops": 4 * pairs * width * case["G"]}
    row = 2 * case["layers"] * width * e  # keys and values of a position, all layers
    if case["kind"] == "step":
        page = case["page"]
        copies = sum(1 for p in z["parent"] if z["held"][p] % page)
        shared = sum(-(-z["held"][p] // page) for p in z["parent"])
        return {"bytes": 2 * copies * page * row + 2 * sum(z["n"]) * row + 4 * (2 * shared + 2 * z["n_pages"] + 8 * case["R"]), "flops": 0}
    # pages above the line in a random arrangement: used * (1 - used / n_pages) of them
    moves = z["used"] * (z["n_pages"] - z["used"]) // z["n_pages"]
    return {"bytes": 2 * moves * case["page"] * row + 4 * (2 * z["slots"] * z["width"] + 2 * z["n_pages"]), "flops": 0}


# ---------------------------------------------------------------------------------- the definition in 64 bits
def exact(case, seed):
    """Attention, request by request and head by head; the other kinds move values and compute none."""
    if case["kind"] != "attend":
        return None
    s = prepare(case, seed)
    table, lens, off, G = s["table"].tolist(), s["lens"].tolist(), s["offsets_host"].tolist(), case["G"]
    out = torch.zeros(s["Q"].shape, dtype=torch.float64, device="cuda")
    for r, slot in enumerate(s["slots"].tolist()):
        a, b, L = off[r], off[r + 1], lens[slot]
        n = b - a
        where = torch.tensor([table[slot][p] * case["page"] + i for p in range(-(-L // case["page"])) for i in range(case["page"])][:L], device="cuda")
        key = torch.arange(L, device="cuda")
        pos = torch.arange(L - n, L, device="cuda") if case["causal"] else torch.full((n,), L, device="cuda")
        mask = torch.zeros((n, L), dtype=torch.bool, device="cuda")
        if case["causal"]:
            mask |= key[None] > pos[:, None]
            if s["prefix"] is not None:
                mask &= key[None] >= int(s["prefix"][r])
        if s["begin"] is not None:
            mask |= key[None] < s["begin"][a:b, None]
        empty = mask.all(1)
        for h in range(case["Hkv"] * G):
            k = s["K"][0].reshape(-1, case["Hkv"], case["dh"])[where, h // G].double()
            v = s["V"][0].reshape(-1, case["Hkv"], case["dh"])[where, h // G].double()
            x = s["Q"][a:b, h].double() @ k.T / math.sqrt(case["dh"])
            if case["cap"]:
                x = case["cap"] * torch.tanh(x / case["cap"])
            if s["slopes"] is not None:
                x = x - s["slopes"][h].double() * (pos[:, None] - key[None]).abs().double()
            x = torch.where(mask, -math.inf, x)
            o = torch.softmax(x, -1) @ v
            out[a:b, h] = torch.where(empty[:, None], 0.0, o)
    return out
