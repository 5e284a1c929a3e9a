"""The KV cache held in pages, as cases that can be timed and compared.

Four operators that a serving stack uses one after the other: rows of K and V go to the pages of their requests (`store`), new
tokens (a decode step's single ones, a chunk of a prompt) or picked ones attend through the page table, all they have before
them or a sliding window beside a few first tokens (`attention`), the attention that every cached token receives is added up
(`mass`), and a context that has grown too long is cut down to the tokens that received most (`evict`).  Head layouts and
context lengths are those of the synthetic workloads (28:4, 32:8, 32:4 heads of 128 channels, 4:4 of 64 in fp32).

With `own` false `run` computes an operator from elementary operations in 32 bits; with `own` true it makes the framework's
calls.  Every pass leaves its state so that the next one computes the same again.
"""
import math
import random

import torch

own = False
DEV = "cuda"
HEADS = {"tiny": (4, 4, 64), "qwen": (28, 4, 128), "llama": (32, 8, 128), "yi": (32, 4, 128)}
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def listed():
    return [
        # a decode step's new row of one request
        dict(name="store-qwen-1-token", op="store", model="qwen", type="bf16", page=16, batch=1, lo=4001, hi=4001, new=1, rows="last"),
        # a chunk of a long prompt
        dict(name="store-llama-8k", op="store", model="llama", type="bf16", page=64, batch=1, lo=32768, hi=32768, new=8192, rows="last"),
        # the small fp32 layer's recomputed tokens
        dict(name="attention-tiny-77", op="attention", model="tiny", type="f32", page=16, batch=1, lo=512, hi=512, new=77, rows="picked", window=0, first=0, idle=0),
        # a decode step of one short request: nothing but latency
        dict(name="attention-qwen-1x601", op="attention", model="qwen", type="bf16", page=16, batch=1, lo=601, hi=601, new=1, rows="last", window=0, first=0, idle=0),
        # a decode step of one long request
        dict(name="attention-yi-1x131k", op="attention", model="yi", type="bf16", page=32, batch=1, lo=131072, hi=131072, new=1, rows="last", window=0, first=0, idle=0),
        # a decode step of a full, ragged batch in which a few requests have ended
        dict(name="attention-llama-64x", op="attention", model="llama", type="bf16", page=16, batch=64, lo=4096, hi=16384, new=1, rows="last", window=0, first=0, idle=3),
        # a chunk of new tokens behind a long reused context
        dict(name="attention-llama-2k-of-32k", op="attention", model="llama", type="bf16", page=64, batch=1, lo=32768, hi=32768, new=2048, rows="last", window=0, first=0, idle=0),
        # a whole prompt under a sliding window, with four first tokens that stay visible
        dict(name="attention-llama-window", op="attention", model="llama", type="bf16", page=16, batch=1, lo=8192, hi=8192, new=8192, rows="last", window=4096, first=4, idle=0),
        # what a decode step adds to every token's attention
        dict(name="mass-llama-64x", op="mass", model="llama", type="bf16", page=16, batch=64, lo=4096, hi=16384, new=1, rows="last", window=0, first=0, idle=3, decay=1.0),
        # and what a chunk adds
        dict(name="mass-llama-2k-of-32k", op="mass", model="llama", type="bf16", page=64, batch=1, lo=32768, hi=32768, new=2048, rows="last", window=0, first=0, idle=0, decay=1.0),
        # a request that has outgrown its share of the cache by a little
        dict(name="evict-qwen-4097", op="evict", model="qwen", type="bf16", page=16, batch=1, lo=4097, hi=4097, keep=3584, first=4, recent=512),
        # a long context cut to its half
        dict(name="evict-yi-131k", op="evict", model="yi", type="bf16", page=32, batch=1, lo=131072, hi=131072, keep=65536, first=4, recent=1024),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["store", "attention", "attention", "attention", "mass", "mass", "evict"])
    model = rng.choice(["tiny", "qwen", "llama", "yi", "llama"])
    c = dict(op=op, model=model, type="f32" if model == "tiny" else "bf16", page=rng.choice([16, 32, 64, 128]))
    most = 4096 if model == "tiny" else 131072 if model == "yi" else 32768
    batch = rng.choice([1, 1, 1, 2, 5]) if op == "evict" else _log(rng, 1, 64)
    if op == "evict":
        hi = _log(rng, 40, most) // (1 if batch == 1 else 4) + 2
        return dict(c, batch=batch, lo=max(1, hi // 2), hi=hi, keep=max(1, int(hi * rng.uniform(0.2, 0.9))), first=rng.choice([0, 1, 4]), recent=_log(rng, 1, max(1, hi // 4)))
    if op == "store":
        hi = min(_log(rng, 16, most), 200000 // batch)
        new = rng.choice([1, 1, _log(rng, 1, max(1, hi // 4))])
        return dict(c, batch=batch, lo=max(new, hi // 2), hi=hi, new=min(new, max(1, 8192 // batch)), rows=rng.choice(["last", "picked"]))
    sight = dict(window=0, first=0)
    if rng.random() < 0.5:                                              # a decode step, now and then of a few tokens a request
        hi = max(8, min(_log(rng, 64, most), 600000 // batch))
        c.update(batch=batch, lo=max(4, hi // 4), hi=hi, new=rng.choice([1, 1, 1, 4]), rows="last", idle=rng.randrange(0, 1 + batch // 8))
    else:
        batch = rng.choice([1, 1, 1, 3, 8])
        hi = max(64, _log(rng, 128, 16384 if model != "tiny" else 2048) // (1 if batch == 1 else 2))
        new = rng.choice([int(hi * math.exp(rng.uniform(math.log(0.02), 0.0))), _log(rng, 5, hi)])
        c.update(batch=batch, lo=max(1, hi // 2), hi=hi, new=max(1, min(new, hi // 2, 4096 // batch)), rows=rng.choice(["last", "last", "picked"]), idle=0)
    if rng.random() < 0.35:
        sight = dict(window=_log(rng, 8, c["hi"]), first=rng.choice([0, 1, 4, 20]))
    c.update(sight)
    if op == "mass":
        c["decay"] = rng.choice([1.0, 1.0, 0.9])
    return c


# ---- inputs ------------------------------------------------------------------------------------------------

def _randn(shape, gen, dtype=torch.float32, scale=1.0):
    return (torch.randn(shape, generator=gen, device=DEV) * scale).to(dtype)


def _table(counts, free, width):
    """Page ids of each request, taken from the list of free pages; entries behind them name no page."""
    t = torch.full((len(counts), width), -1, dtype=torch.int32, device=DEV)
    at = 0
    for b, n in enumerate(counts):
        t[b, :n] = free[at:at + n]
        at += n
    return t


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    rng = random.Random(seed)
    op, page, batch = case["op"], case["page"], case["batch"]
    hq, hk, d = HEADS[case["model"]]
    dt = TYPES[case["type"]]
    lens = [rng.randint(case["lo"], case["hi"]) for _ in range(batch)]
    pages = [-(-n // page) for n in lens]
    width = -(-case["hi"] // page)
    kept = [-(-min(n, case["keep"]) // page) for n in lens] if op == "evict" else []
    n_pages = batch * width + (batch * -(-case["keep"] // page) if op == "evict" else 0) + 3     # of any lengths
    free = torch.randperm(n_pages, generator=gen, device=DEV).to(torch.int32)
    s = {"case": case, "lens": lens, "table": _table(pages, free, width), "ctx_len": torch.tensor(lens, dtype=torch.int32, device=DEV)}
    s["k"], s["v"] = (_randn((n_pages, page, hk, d), gen, dt) for _ in range(2))
    if own:
        from paper_2503_16525_amd import binding as kvs
        s["shape"] = kvs.make_shape(hq, hk, d, kvs.BF16 if case["type"] == "bf16" else kvs.F32)
        s["cache"] = kvs.PagedCache(s["k"], s["v"])
        s["pages"] = kvs.PageTable(s["table"], s["ctx_len"], case["hi"])
    if op == "evict":
        width = -(-case["keep"] // page)
        s["new_table"] = _table(kept, free[sum(pages):], width)
        # whole steps of 2^-10, at most 2^10: sums over the heads have no rounding, and ties come up
        w = torch.exp(_randn((batch, hk, case["hi"]), gen) * 2.0 - 1.0).clamp_max(1024.0)
        s["mass"] = (w * 1024.0).round() / 1024.0
        s["keep"] = torch.full((batch,), case["keep"], dtype=torch.int32, device=DEV)
        s["kept"] = torch.full((batch, case["keep"]), -1, dtype=torch.int32, device=DEV)
        s["new_len"] = torch.zeros((batch,), dtype=torch.int32, device=DEV)
        s["new_mass"] = torch.zeros((batch, hk, case["keep"]), device=DEV)
        if own:
            size = kvs.kvs_workspace_size("evict_paged", s["shape"], batch, case["hi"], 0)
            s["ws"] = torch.empty((size,), dtype=torch.uint8, device=DEV)
        return s
    new = [min(case["new"], n) for n in lens]
    cu = [0]
    for n in new:
        cu.append(cu[-1] + n)
    s["cu"] = torch.tensor(cu, dtype=torch.int32, device=DEV)
    s["new"], s["n"], s["start"] = new, cu[-1], cu
    s["pos"] = None
    if case["rows"] == "picked":
        s["pos"] = torch.tensor(sum((sorted(rng.sample(range(n), m)) for n, m in zip(lens, new)), []), dtype=torch.int32, device=DEV)
    # request of every token, and its place among that request's
    s["of"] = torch.tensor([b for b, m in enumerate(new) for _ in range(m)], device=DEV)
    s["place"] = torch.tensor([i for m in new for i in range(m)], device=DEV)
    s["count"] = torch.tensor(new, device=DEV)
    if case["new"] == 1:
        s["cu"] = None                                                  # one token a request
    if op == "store":
        s["k_new"], s["v_new"] = (_randn((s["n"], hk, d), gen, dt) for _ in range(2))
        s["mass"] = torch.rand((batch, hk, case["hi"]), generator=gen, device=DEV)
        return s
    for b in rng.sample(range(batch), case["idle"]):                    # ended requests keep their place in the batch
        s["lens"][b] = 0
    s["ctx_len"].copy_(torch.tensor(lens, dtype=torch.int32))
    s["q"] = _randn((s["n"], hq, d), gen, dt)
    s["scale"] = d ** -0.5
    if op == "attention":
        s["out"], s["lse"] = torch.empty_like(s["q"]), torch.empty((s["n"], hq), device=DEV)
    else:
        s["lse"] = _plain_attention(s, False)[0]
        s["mass"] = torch.rand((batch, hk, case["hi"]), generator=gen, device=DEV)
        s["mass_out"] = s["mass"].clone()
    if own:
        size = kvs.kvs_workspace_size(op + "_paged", s["shape"], batch, case["hi"], s["n"])
        s["ws"] = torch.empty((size,), dtype=torch.uint8, device=DEV)
    return s


# ---- one pass ----------------------------------------------------------------------------------------------

def run(state):
    s, case = state, state["case"]
    if own:
        from paper_2503_16525_amd import binding as kvs
    if case["op"] == "store":
        if own:
            kvs.kvs_store_paged(s["shape"], s["cache"], s["pages"], s["cu"], s["pos"], s["k_new"], s["v_new"], s["mass"])
        else:
            _plain_store(s)
        return [s["k"], s["v"], s["mass"]]
    if case["op"] == "attention":
        if own:
            kvs.kvs_attention_paged(s["shape"], s["cache"], s["pages"], s["cu"], s["pos"], s["q"], s["scale"], case["window"], case["first"], s["out"], s["lse"], s["ws"])
            return [s["out"], s["lse"]]
        return _plain_attention(s, True)
    if case["op"] == "mass":
        if own:
            kvs.kvs_mass_paged(s["shape"], s["cache"], s["pages"], s["cu"], s["pos"], s["q"], s["lse"], s["scale"], case["window"], case["first"], case["decay"],
                               s["mass"], s["mass_out"], s["ws"])
        else:
            _plain_mass(s)
        return [s["mass_out"]]
    if own:
        kvs.kvs_evict_paged(s["shape"], s["cache"], s["pages"], s["keep"], case["first"], case["recent"], s["mass"], s["new_table"], s["kept"], s["new_len"], s["new_mass"], s["ws"])
    else:
        _plain_evict(s)
    return [s["k"], s["v"], s["kept"], s["new_len"], s["new_mass"]]


def _positions(s):
    if s["pos"] is not None:
        return s["pos"].long()
    return (s["ctx_len"] - s["count"])[s["of"]] + s["place"]


def _plain_store(s):
    page = s["case"]["page"]
    of, pos = s["of"], _positions(s)
    slot = s["table"][of, pos // page].long() * page + pos % page
    for x in ("k", "v"):
        s[x].flatten(0, 1)[slot] = s[x + "_new"]
    s["mass"][of, :, pos] = 0.0


def _scores(s, b0, b1):
    """Scores of requests b0 .. b1 - 1 [requests, KV heads, tokens * query heads a KV head, keys], what no token sees at -inf, the
    tokens in their rows, and the keys' places in the pool."""
    case = s["case"]
    hq, hk, d = HEADS[case["model"]]
    grp, page, nb = hq // hk, case["page"], b1 - b0
    longest, most = max(max(s["lens"][b0:b1]), 1), max(s["new"][b0:b1])
    key = torch.arange(longest, device=DEV)
    slot = s["table"][b0:b1][:, key // page].clamp_min(0).long() * page + key % page
    place = torch.arange(most, device=DEV)
    count, length = s["count"][b0:b1], s["ctx_len"][b0:b1, None, None]
    token = ((count.cumsum(0) - count)[:, None] + s["start"][b0] + place).clamp_max(s["n"] - 1)      # [requests, most]
    pos = _positions(s)[token]
    seen = (key <= pos[:, :, None]) & (key < length) & (place < count[:, None])[:, :, None]
    if case["window"] > 0:
        seen &= (key > pos[:, :, None] - case["window"]) | (key < case["first"])
    q = s["q"][token].float().view(nb, most, hk, grp, d).permute(0, 2, 1, 3, 4).reshape(nb, hk, most * grp, d)
    k = s["k"].flatten(0, 1)[slot].float().permute(0, 2, 3, 1).contiguous()             # [requests, hk, d, keys]
    score = torch.matmul(q, k).mul_(s["scale"])
    score.view(nb, hk, most, grp, longest).masked_fill_(~seen[:, None, :, None, :], -math.inf)
    return score, token, slot


def _groups(s):
    """Requests that are computed together: as many as a few gigabytes of scores hold."""
    hq = HEADS[s["case"]["model"]][0]
    b = 0
    while b < len(s["lens"]):
        e = b + 1
        while e < len(s["lens"]) and (e + 1 - b) * max(s["lens"][b:e + 1]) * max(hq * max(s["new"][b:e + 1]), 4096) < 1 << 32:
            e += 1
        yield b, e
        b = e


def _plain_attention(s, values):
    case = s["case"]
    hq, hk, d = HEADS[case["model"]]
    grp = hq // hk
    out, lse = torch.empty_like(s["q"]), torch.empty((s["n"], hq), device=DEV)
    for b0, b1 in _groups(s):
        score, _, slot = _scores(s, b0, b1)
        nb, rows = score.shape[0], score.shape[2] // grp
        mine = slice(s["start"][b0], s["start"][b1])
        top = score.amax(-1, keepdim=True).clamp_min(-3e38)
        score.sub_(top).exp_()
        total = score.sum(-1, keepdim=True)
        per_token = lambda x: x.view(nb, hk, rows, grp, -1).permute(0, 2, 1, 3, 4).reshape(nb, rows, hq, -1)[s["of"][mine] - b0, s["place"][mine]]
        lse[mine] = per_token(torch.where(total > 0, top + total.log(), torch.full_like(top, -math.inf)))[..., 0]
        if values:
            v = s["v"].flatten(0, 1)[slot].float().permute(0, 2, 1, 3).contiguous()
            x = torch.matmul(score, v)
            out[mine] = per_token(torch.where(total > 0, x / total, torch.zeros_like(x))).to(out.dtype)
    return [out, lse] if values else [lse]


def _plain_mass(s):
    case = s["case"]
    hq, hk, d = HEADS[case["model"]]
    grp = hq // hk
    for b0, b1 in _groups(s):
        score, token, _ = _scores(s, b0, b1)
        nb, rows, longest = score.shape[0], score.shape[2] // grp, score.shape[3]
        lse = s["lse"][token].view(nb, rows, hk, grp).permute(0, 2, 1, 3).reshape(nb, hk, rows * grp, 1)
        lse = torch.where(torch.isfinite(lse), lse, torch.zeros_like(lse))              # tokens that see nothing: every score is -inf
        got = score.sub_(lse).exp_().sum(2)
        old = s["mass"][b0:b1, :, :longest]
        inside = torch.arange(longest, device=DEV) < s["ctx_len"][b0:b1, None]
        s["mass_out"][b0:b1, :, :longest] = torch.where(inside[:, None], old * case["decay"] + got, s["mass_out"][b0:b1, :, :longest])


def _plain_evict(s):
    case = s["case"]
    page = case["page"]
    for b, n in enumerate(s["lens"]):
        m = min(n, case["keep"])
        weight = s["mass"][b, 0, :n].clone()
        for g in range(1, s["mass"].shape[1]):
            weight += s["mass"][b, g, :n]
        at = torch.arange(n, device=DEV)
        first, recent = min(case["first"], m), min(case["recent"], m - min(case["first"], m))
        weight[(at < first) | (at >= n - recent)] = math.inf
        order = torch.sort(weight, descending=True, stable=True).indices
        keep = torch.sort(order[:m]).values
        to = torch.arange(m, device=DEV)
        slot = s["table"][b, keep // page].long() * page + keep % page
        into = s["new_table"][b, to // page].long() * page + to % page
        for x in ("k", "v"):
            rows = s[x].flatten(0, 1)
            rows[into] = rows[slot]
        s["kept"][b, :m] = keep.to(torch.int32)
        s["new_mass"][b, :, :m] = s["mass"][b][:, keep]
        s["new_len"][b] = m


# ---- what a pass cannot do without, and its results in 64 bits ---------------------------------------------

def _seen(case):
    """Keys that a token sees, and keys that a request's tokens see between them, on average."""
    length, new = 0.5 * (case["lo"] + case["hi"]), case["new"]
    w, f = case["window"], case["first"]
    count = lambda p: min(p + 1.0, w + min(f, max(p + 1.0 - w, 0.0))) if w else p + 1.0
    lowest = 0.0 if case["rows"] == "picked" else length - new
    steps = 64
    at = [lowest + (length - lowest) * (i + 0.5) / steps for i in range(steps)] if new > 1 or case["rows"] == "picked" else [length - 1.0]
    mean = sum(count(p) for p in at) / len(at)
    if case["rows"] == "picked":                                        # windows that cover what lies between the tokens
        reach = min(length * new / (new + 1.0), (w + f) * new) if w else length * new / (new + 1.0)
    else:
        reach = min(length, w + new - 1.0 + f) if w else length
    return mean, reach


def work(case):
    hq, hk, d = HEADS[case["model"]]
    e = 2 if case["type"] == "bf16" else 4
    length = 0.5 * (case["lo"] + case["hi"])
    if case["op"] == "evict":
        m = min(case["keep"], length)
        return {"bytes": case["batch"] * (4.0 * hk * (length + m) + m * (4 * hk * d * e + 4) + 4.0 * (length + m) / case["page"]), "flops": 1.0 * case["batch"] * length * hk}
    rows = case["batch"] * min(case["new"], length)
    if case["op"] == "store":
        return {"bytes": rows * (4 * hk * d * e + 4 * hk + (8 if case["rows"] == "picked" else 4)), "flops": 0.0}
    live = case["batch"] - case["idle"]
    mean, reach = _seen(case)
    table = 4.0 * live * reach / case["page"]
    dots = 2.0 * d * hq * live * min(case["new"], length) * mean
    if case["op"] == "attention":
        return {"bytes": live * reach * 2 * hk * d * e + rows * hq * (2 * d * e + 4) + table, "flops": 2 * dots}
    return {"bytes": live * (reach * hk * d * e + length * hk * 8) + rows * hq * (d * e + 4) + table, "flops": dots}


def exact(case, seed):
    s = prepare(case, seed)
    hq, hk, d = HEADS[case["model"]]
    page = case["page"]
    if case["op"] == "store":                                           # nothing but copies
        k, v, mass = s["k"].double(), s["v"].double(), s["mass"].double()
        for b, n in enumerate(s["lens"]):
            mine = slice(s["start"][b], s["start"][b + 1])
            p = torch.arange(n - s["new"][b], n, device=DEV) if s["pos"] is None else s["pos"][mine].long()
            to = s["table"][b].long()[torch.div(p, page, rounding_mode="floor")]
            k[to, p.remainder(page)], v[to, p.remainder(page)] = s["k_new"][mine].double(), s["v_new"][mine].double()
            mass[b] = mass[b].index_fill(1, p, 0.0)
        return [k, v, mass]
    if case["op"] == "evict":
        return _exact_evict(s)
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
    lse = torch.full((s["n"], hq), -math.inf, dtype=torch.float64, device=DEV)
    mass = s["mass_out"].double() if case["op"] == "mass" else None
    for b, n in enumerate(s["lens"]):
        mine = slice(s["start"][b], s["start"][b + 1])
        if mass is not None:
            mass[b, :, :n] = s["mass"][b, :, :n].double() * case["decay"]
        if n == 0:
            continue
        i = torch.arange(n, device=DEV)
        p = (s["pos"][mine].long() if s["pos"] is not None else torch.arange(n - s["new"][b], n, device=DEV))[:, None]
        visible = i <= p
        if case["window"]:
            visible &= torch.logical_or(p - i < case["window"], i < case["first"])
        rows = (s["table"][b].long()[torch.div(i, page, rounding_mode="floor")], i.remainder(page))
        for g in range(hk):
            k, v = s["k"][rows[0], rows[1], g].double(), s["v"][rows[0], rows[1], g].double()
            for h in range(g * (hq // hk), (g + 1) * (hq // hk)):
                logit = torch.where(visible, s["scale"] * (s["q"][mine, h].double() @ k.T), -math.inf)
                if mass is None:
                    lse[mine, h] = torch.logsumexp(logit, 1)
                    out[mine, h] = torch.where(visible.any(1, keepdim=True), torch.softmax(logit, 1) @ v, 0.0)
                else:
                    mass[b, g, :n] += torch.where(visible, torch.exp(logit - s["lse"][mine, h].double()[:, None]), 0.0).sum(0)
    return [out, lse] if mass is None else [mass]


def _exact_evict(s):
    case = s["case"]
    page, m_most = case["page"], case["keep"]
    k, v = s["k"].double(), s["v"].double()
    kept, new_len, new_mass = s["kept"].long(), s["new_len"].long(), s["new_mass"].double()
    for b, n in enumerate(s["lens"]):
        m = min(n, m_most)
        safe = list(range(min(case["first"], m)))
        safe += list(range(max(n - case["recent"], n - (m - len(safe)), len(safe)), n))
        free = torch.ones((n,), dtype=torch.bool, device=DEV)
        free[torch.tensor(safe, dtype=torch.long, device=DEV)] = False
        others = free.nonzero()[:, 0]
        weight = s["mass"][b].double().sum(0)[others]
        # by weight, then by place: two stable passes from the last key to the first
        ranked = others[torch.argsort(-weight, stable=True)][: m - len(safe)]
        mine = torch.cat((ranked, torch.tensor(safe, dtype=torch.long, device=DEV))).sort().values
        to = torch.arange(m, device=DEV)
        src = (s["table"][b].long()[torch.div(mine, page, rounding_mode="floor")], mine.remainder(page))
        dst = (s["new_table"][b].long()[torch.div(to, page, rounding_mode="floor")], to.remainder(page))
        k[dst], v[dst] = s["k"][src].double(), s["v"][src].double()
        kept[b, :m], new_len[b] = mine, m
        new_mass[b, :, :m] = s["mass"][b].double()[:, mine]
    return [k, v, kept, new_len, new_mass]
