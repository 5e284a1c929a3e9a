"""The KV cache held in 8 bits and the rotary positions of what is reused from it, as cases that can be timed and compared.

Four operators that a serving stack uses one after the other: a reused key is turned to the position that it takes in
the new request (`rotary`), rows of K and V are stored in 8 bits with a scale for each block of tokens and KV head
(`store`), the deviation of the freshly computed values from what the cache holds ranks the reused tokens (`deviation`),
and the picked tokens, or a decode step's single ones, attend over the cache (`attention`).  Head layouts and context
lengths are those of the synthetic workloads (28:4, 32:8, 32:4 heads of 128 channels, 4:4 of 64 in fp32).

With `own` false `run` computes an operator from elementary operations in 32 bits (angles in 64); with `own` true it
makes the framework's calls.  Every pass leaves its state so that the next one computes the same again.
"""
import math
import random

import torch

own = False
DEV = "cuda"
HEADS = {"tiny": (4, 4, 64), "qwen": (28, 4, 128), "llama": (32, 8, 128), "yi": (32, 4, 128)}
CODES = {"e4m3": torch.float8_e4m3fn, "int8": torch.int8}
TOP = {"e4m3": 448.0, "int8": 127.0}
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
LEAST = 2.0 ** -126     # the smallest scale of a block that holds anything but zeros


def listed():
    return [
        # the smallest call: one decode step's token, far into a long context
        dict(name="rotary-1-token", op="rotary", model="qwen", type="bf16", n=1, layout="half", part=128, scaling="plain", move=False, far=100000, fused=True),
        # a prompt's Q and K out of the fused projection's buffer, positions stretched by wavelength
        dict(name="rotary-llama-8k", op="rotary", model="llama", type="bf16", n=8192, layout="half", part=128, scaling="wavelength", move=False, far=8192, fused=True),
        # reused keys moved to their places in a new request; neighbouring channels paired, half of the head turned
        dict(name="rotary-move-yi-131k", op="rotary", model="yi", type="bf16", n=131072, layout="interleaved", part=64, scaling="ramp", move=True, far=131072, fused=False),
        # the small fp32 layer's whole prompt into the cache
        dict(name="store-tiny-int8", op="store", model="tiny", type="f32", code="int8", block=16, n_rows=512, n=512, rows="whole"),
        # what a layer recomputes of a 32k context (15 %), written over the reused rows
        dict(name="store-llama-4424", op="store", model="llama", type="bf16", code="e4m3", block=32, n_rows=32768, n=4424, rows="picked"),
        # a long prompt into the cache
        dict(name="store-yi-131k", op="store", model="yi", type="bf16", code="int8", block=128, n_rows=131072, n=131072, rows="whole"),
        # the check layer's scores of a request of ordinary, odd length, keys among them
        dict(name="deviation-qwen-6001", op="deviation", model="qwen", type="bf16", code="int8", block=64, n=6001, mode="kv", alpha=True),
        # and of a long prompt, values only
        dict(name="deviation-llama-32k", op="deviation", model="llama", type="bf16", code="e4m3", block=32, n=32768, mode="v", alpha=False),
        # the small fp32 layer's recomputed tokens
        dict(name="attention-tiny-77", op="attention", model="tiny", type="f32", code="int8", block=16, batch=1, lo=512, hi=512, rows=77, idle=0),
        # a decode step of one long request
        dict(name="attention-yi-1x131k", op="attention", model="yi", type="bf16", code="int8", block=64, batch=1, lo=131072, hi=131072, rows=1, idle=0),
        # a decode step of a full, ragged batch in which a few requests have ended
        dict(name="attention-llama-64x", op="attention", model="llama", type="bf16", code="e4m3", block=32, batch=64, lo=4096, hi=16384, rows=1, idle=3),
        # the recomputed tokens of a long prompt
        dict(name="attention-llama-32k", op="attention", model="llama", type="bf16", code="e4m3", block=32, batch=1, lo=32768, hi=32768, rows=4424, idle=0),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["rotary", "store", "deviation", "attention", "attention"])
    model = rng.choice(["tiny", "qwen", "llama", "yi", "llama"])
    kind = "f32" if model == "tiny" else "bf16"
    code, block = rng.choice(["e4m3", "int8"]), rng.choice([16, 32, 64, 128])
    most = 4096 if model == "tiny" else 131072 if model == "yi" else 32768
    if op == "rotary":
        far = _log(rng, 1000, 1000000)
        return dict(op=op, model=model, type=kind, n=_log(rng, 1, most), layout=rng.choice(["half", "interleaved"]),
                    part=rng.choice([32, 64]) if model == "tiny" else rng.choice([32, 64, 96, 128]),
                    scaling=rng.choice(["plain", "linear", "ntk", "ramp", "wavelength"]), move=rng.random() < 0.3, far=far, fused=rng.random() < 0.5)
    if op == "store":
        n_rows = _log(rng, 16, most)
        rows = rng.choice(["whole", "picked", "picked", "appended"])
        n = n_rows if rows == "whole" else min(n_rows, _log(rng, 1, 64)) if rows == "appended" else max(1, int(n_rows * rng.uniform(0.02, 0.30)))
        return dict(op=op, model=model, type=kind, code=code, block=block, n_rows=n_rows, n=n, rows=rows)
    if op == "deviation":
        return dict(op=op, model=model, type=kind, code=code, block=block, n=_log(rng, 64, most), mode=rng.choice(["v", "v", "kv"]), alpha=rng.random() < 0.5)
    if rng.random() < 0.5:                                              # a decode step, now and then of a few tokens a request
        batch = _log(rng, 1, 64)
        hi = min(_log(rng, 64, most), 1000000 // batch)
        return dict(op=op, model=model, type=kind, code=code, block=block, batch=batch, lo=max(1, hi // 4), hi=hi, rows=min(rng.choice([1, 1, 1, 4]), max(1, hi // 4)),
                    idle=rng.randrange(0, 1 + batch // 8))
    batch = rng.choice([1, 1, 1, 3, 8])
    hi = _log(rng, 128, 16384 if model != "tiny" else 2048) // (1 if batch == 1 else 2)
    return dict(op=op, model=model, type=kind, code=code, block=block, batch=batch, lo=max(1, hi // 2), hi=hi,
                rows=max(1, int(hi // 2 * math.exp(rng.uniform(math.log(0.02), math.log(0.30))))), idle=0)


# ---- inputs ------------------------------------------------------------------------------------------------

def _randn(shape, gen, dtype=torch.float32, scale=1.0):
    return (torch.randn(shape, generator=gen, device=DEV) * scale).to(dtype)


def _kv(n, case, gen):
    """Values as another request left them: unit normal with a noise of its own for each token."""
    hk, d = HEADS[case["model"]][1:]
    sigma = torch.exp(_randn((n, 1, 1), gen) * 1.0 - 3.0)
    return _randn((n, hk, d), gen) * (1.0 + sigma)


def _encode(y, code):
    return y.round().clamp(-127, 127).to(torch.int8) if code == "int8" else y.clamp(-448.0, 448.0).to(torch.float8_e4m3fn)


def _filled(x, case):
    """A cache that holds x [n, heads, channels]: codes and scales."""
    n, hk, d = x.shape
    blk = case["block"]
    nb = -(-n // blk)
    pad = torch.zeros((nb * blk, hk, d), device=DEV)
    pad[:n] = x
    scale = pad.view(nb, blk, hk, d).abs().amax(dim=(1, 3)) / TOP[case["code"]]
    inv = torch.where(scale > 0, 1.0 / scale, torch.zeros_like(scale))
    return _encode(x * inv.repeat_interleave(blk, 0)[:n, :, None], case["code"]), scale


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    rng = random.Random(seed)
    hq, hk, d = HEADS[case["model"]]
    dt = TYPES[case["type"]]
    s = {"case": case}
    if case["op"] == "rotary":
        n = case["n"]
        if case["fused"]:                                               # slices of one buffer of Q, K and V rows
            buf = _randn((n, hq + 2 * hk, d), gen, dt)
            s["q"], s["k"] = buf[:, :hq], buf[:, hq:hq + hk]
        else:
            s["q"], s["k"] = _randn((n, hq, d), gen, dt), _randn((n, hk, d), gen, dt)
        if case["move"]:                                                # keys alone; spans of the earlier request
            s["q"] = None
            s["pos_from"] = torch.randint(0, case["far"], (n,), generator=gen, device=DEV, dtype=torch.int32)
        else:
            s["pos_from"] = None
        first = rng.randrange(0, max(1, case["far"] - n))
        s["pos"] = torch.arange(first, first + n, device=DEV, dtype=torch.int32)
        s["q_out"] = None if case["move"] else torch.empty((n, hq, d), dtype=dt, device=DEV)
        s["k_out"] = torch.empty((n, hk, d), dtype=dt, device=DEV)
        if own:
            from paper_2503_16525_amd import binding as kvs
            s["shape"] = kvs.make_shape(hq, hk, d, kvs.BF16 if case["type"] == "bf16" else kvs.F32)
            s["spec"] = kvs.rotary_spec(**_rotary_args(case))
        return s
    n_rows = case.get("n_rows", case.get("n", 0))
    if case["op"] == "attention":
        lens = [rng.randint(case["lo"], case["hi"]) for _ in range(case["batch"])]
        off = [0]
        for n in lens:                                                  # each request's rows begin with a block of its own
            off.append(-(-(off[-1] + n) // case["block"]) * case["block"])
        n_rows = off[-1]
    for x in ("k", "v"):
        s[x], s[x + "_scale"] = _filled(_kv(n_rows, case, gen), case)
    if own:
        from paper_2503_16525_amd import binding as kvs
        s["shape"] = kvs.make_shape(hq, hk, d, kvs.BF16 if case["type"] == "bf16" else kvs.F32)
        s["cache"] = kvs.Cache8(s["k"], s["v"], s["k_scale"], s["v_scale"], case["block"])
    if case["op"] == "store":
        n = case["n"]
        s["k_new"], s["v_new"] = _randn((n, hk, d), gen, dt), _randn((n, hk, d), gen, dt)
        if case["rows"] == "whole":
            s["pos"] = None
        else:
            s["pos"] = torch.randperm(n_rows, generator=gen, device=DEV)[:n].sort().values.to(torch.int32)
        s["reused"] = torch.ones((n_rows,), dtype=torch.uint8, device=DEV)
        s["dev_v"] = torch.rand((hk, n_rows), generator=gen, device=DEV)
    elif case["op"] == "deviation":
        n = case["n"]
        for x in ("k", "v"):                                            # what the layer computes afresh lies near what the cache holds
            sigma = torch.exp(_randn((n, 1, 1), gen) * 1.5 - 3.0)
            held = s[x].float() * s[x + "_scale"].repeat_interleave(case["block"], 0)[:n, :, None]
            s[x + "_fresh"] = (held + sigma * _randn((n, hk, d), gen)).to(dt)
        s["reused"] = (torch.rand((n,), generator=gen, device=DEV) < 0.9).to(torch.uint8)
        s["alpha"] = torch.rand((hk, n), generator=gen, device=DEV) + 0.5 if case["alpha"] else None
        s["dev_v"], s["score"] = torch.empty((hk, n), device=DEV), torch.empty((n,), device=DEV)
        s["dev_k"] = torch.empty((hk, n), device=DEV) if case["mode"] == "kv" else None
    else:
        rows = case["rows"]
        s["ctx_off"], s["ctx_len"], s["cu_sel"] = off[:-1], lens, [rows * b for b in range(len(lens) + 1)]
        pos = [sorted(rng.sample(range(n), rows)) if rows > 4 else list(range(n - rows, n)) for n in lens]
        for b in rng.sample(range(len(lens)), case["idle"]):            # ended requests keep their place in the batch
            pos[b] = [-1] * rows
        s["pos"] = torch.tensor(sum(pos, []), dtype=torch.int32, device=DEV)
        s["q"] = _randn((rows * len(lens), hq, d), gen, dt, d ** -0.5)
        s["out"] = torch.empty_like(s["q"])
        s["lse"] = torch.empty((rows * len(lens), hq), device=DEV)
        if own:
            size = kvs.kvs_workspace_size("attention_kv8", s["shape"], len(lens), n_rows, rows * len(lens))
            s["ws"] = torch.empty((size,), dtype=torch.uint8, device=DEV)
    return s


# ---- one pass ----------------------------------------------------------------------------------------------

def run(state):
    s, case = state, state["case"]
    if own:
        from paper_2503_16525_amd import binding as kvs
    if case["op"] == "rotary":
        if own:
            kvs.kvs_rotary(s["shape"], s["spec"], s["pos"], s["pos_from"], s["q"], s["k"], s["q_out"], s["k_out"])
            return [x for x in (s["q_out"], s["k_out"]) if x is not None]
        return _plain_rotary(s)
    if case["op"] == "store":
        if own:
            kvs.kvs_store_kv8(s["shape"], s["cache"], s["k_new"], s["v_new"], s["pos"], 0, s["reused"], s["dev_v"])
        else:
            _plain_store(s)
        return [s["k"], s["v"], s["k_scale"], s["v_scale"], s["reused"], s["dev_v"]]
    if case["op"] == "deviation":
        if own:
            kvs.kvs_deviation_kv8(s["shape"], s["cache"], 0, case["n"], s["k_fresh"], s["v_fresh"], s["reused"], s["alpha"],
                                  kvs.SCORE_KV if case["mode"] == "kv" else kvs.SCORE_V, s["dev_k"], s["dev_v"], s["score"])
            return [x for x in (s["dev_k"], s["dev_v"], s["score"]) if x is not None]
        return _plain_deviation(s)
    if own:
        kvs.kvs_attention_kv8(s["shape"], s["cache"], s["ctx_off"], s["ctx_len"], s["cu_sel"], s["q"], s["pos"], 1.0, s["out"], s["lse"], s["ws"])
        return [s["out"], s["lse"]]
    return _plain_attention(s)


def _rotary_args(case):
    """base and scaling of the frequencies, as the operator takes them"""
    return dict(rotary_dim=case["part"], layout=case["layout"], scaling=case["scaling"], base=500000.0, factor=1.0 if case["scaling"] == "plain" else 8.0,
                original=8192, low=1.0, high=32.0 if case["scaling"] == "ramp" else 4.0,
                magnitude=0.1 * math.log(8.0) + 1.0 if case["scaling"] == "ramp" and not case["move"] else 1.0)


def _frequencies(a):
    """Radians a position of every pair of channels, in 64 bits on the device."""
    r, base, factor = a["rotary_dim"], a["base"], a["factor"]
    j = torch.arange(r // 2, device=DEV, dtype=torch.float64)
    if a["scaling"] == "ntk":
        base = base * factor ** (r / (r - 2))
    f = torch.exp(j * (-2.0 * math.log(base) / r))
    if a["scaling"] == "linear":
        f = f / factor
    if a["scaling"] == "ramp":
        at = lambda turns: r * math.log(a["original"] / (turns * 2 * math.pi)) / (2 * math.log(base))
        lo, hi = max(math.floor(at(a["high"])), 0), min(math.ceil(at(a["low"])), r - 1)
        w = ((j - lo) / max(hi - lo, 0.001)).clamp(0, 1)
        f = f * (1 - w) + f / factor * w
    if a["scaling"] == "wavelength":
        turns = a["original"] * f / (2 * math.pi)
        w = ((turns - a["low"]) / (a["high"] - a["low"])).clamp(0, 1)
        f = f * w + f / factor * (1 - w)
    return f


def _plain_rotary(s):
    a = _rotary_args(s["case"])
    p = s["pos"].double() - (s["pos_from"].double() if s["pos_from"] is not None else 0)
    angle = p[:, None] * _frequencies(a)
    cos, sin = (angle.cos() * a["magnitude"]).float()[:, None], (angle.sin() * a["magnitude"]).float()[:, None]
    r, h = a["rotary_dim"], a["rotary_dim"] // 2
    out = []
    for x in (s["q"], s["k"]):
        if x is None:
            continue
        y = x.float()
        u, v = (y[..., 0:r:2], y[..., 1:r:2]) if a["layout"] == "interleaved" else (y[..., :h], y[..., h:r])
        uu, vv = u * cos - v * sin, v * cos + u * sin
        turned = torch.stack((uu, vv), -1).flatten(-2) if a["layout"] == "interleaved" else torch.cat((uu, vv), -1)
        out.append(torch.cat((turned, y[..., r:]), -1).to(x.dtype))
    return out


def _plain_store(s):
    case = s["case"]
    n_rows, blk, code, top = case["n_rows"], case["block"], case["code"], TOP[case["code"]]
    pos = torch.arange(case["n"], device=DEV) if s["pos"] is None else s["pos"].long()
    at = pos // blk
    nb, row_block = -(-n_rows // blk), torch.arange(n_rows, device=DEV) // blk
    rows_of = torch.zeros((nb,), device=DEV).scatter_add_(0, row_block, torch.ones((n_rows,), device=DEV))
    full = (torch.zeros((nb,), device=DEV).scatter_add_(0, at, torch.ones((case["n"],), device=DEV)) == rows_of)[:, None]
    for x in ("k", "v"):
        new, old = s[x + "_new"].float(), s[x + "_scale"]
        most = torch.zeros_like(old).scatter_reduce_(0, at[:, None].expand(-1, old.shape[1]), new.abs().amax(-1), "amax")
        mine = torch.where(most > 0, torch.clamp_min(most / top, LEAST), torch.zeros_like(most))
        scale = torch.where(full, mine, torch.maximum(old, mine))
        inv = torch.where(scale > 0, 1.0 / scale, torch.zeros_like(scale))
        ratio = torch.where(scale > 0, old / scale, torch.ones_like(scale))
        held = _encode(s[x].float() * ratio[row_block][:, :, None], code).view(torch.uint8)
        held[pos] = _encode(new * inv[at][:, :, None], code).view(torch.uint8)
        s[x].view(torch.uint8).copy_(held)
        s[x + "_scale"].copy_(scale)
    s["reused"][pos] = 0
    s["dev_v"][:, pos] = 0.0


def _plain_deviation(s):
    case, dev = s["case"], {}
    for x in ("k", "v"):
        if s["dev_" + x] is not None:
            held = s[x].float() * s[x + "_scale"].repeat_interleave(case["block"], 0)[: case["n"], :, None]
            dev[x] = (s[x + "_fresh"].float() - held).abs().sum(-1).t().contiguous()
    score = dev["v"] + dev["k"] if case["mode"] == "kv" else dev["v"]
    score = (score * s["alpha"] if s["alpha"] is not None else score).sum(0)
    score = torch.where(s["reused"] != 0, score, torch.full_like(score, -math.inf))
    return [dev[x] for x in ("k", "v") if x in dev] + [score]


def _plain_attention(s):
    case = s["case"]
    hq, hk, d = HEADS[case["model"]]
    grp, rows, batch, longest = hq // hk, case["rows"], case["batch"], max(s["ctx_len"])
    off = torch.tensor(s["ctx_off"], device=DEV)
    key = torch.arange(longest, device=DEV)
    at = (off[:, None] + key).clamp_max(s["k"].shape[0] - 1)            # [batch, longest] cache rows, those behind a context masked below
    held = {}
    for x in ("k", "v"):
        codes = s[x].view(torch.uint8)[at].view(s[x].dtype).float()
        held[x] = codes * s[x + "_scale"][at // case["block"]][..., None]   # [batch, longest, hk, d]
    q = s["q"].float().view(batch, rows, hk, grp, d).permute(0, 2, 1, 3, 4).reshape(batch, hk, rows * grp, d)
    score = torch.matmul(q, held["k"].permute(0, 2, 3, 1).contiguous())
    pos = s["pos"].view(batch, 1, rows, 1, 1).expand(-1, hk, -1, grp, -1).reshape(batch, hk, rows * grp, 1)
    score.masked_fill_(key > pos, -math.inf)
    top = score.amax(-1, keepdim=True).clamp_min(-3e38)
    score.sub_(top).exp_()
    total = score.sum(-1, keepdim=True)
    out = torch.matmul(score, held["v"].permute(0, 2, 1, 3).contiguous())
    out = torch.where(total > 0, out / total, torch.zeros_like(out))
    lse = torch.where(total > 0, top + total.log(), torch.full_like(top, -math.inf))
    out = out.view(batch, hk, rows, grp, d).permute(0, 2, 1, 3, 4).reshape(batch * rows, hq, d)
    lse = lse.view(batch, hk, rows, grp).permute(0, 2, 1, 3).reshape(batch * rows, hq)
    return [out.to(s["q"].dtype), lse.contiguous()]


# ---- what a pass cannot do without, and its results in 64 bits ---------------------------------------------

def work(case):
    hq, hk, d = HEADS[case["model"]]
    e = 2 if case["type"] == "bf16" else 4
    if case["op"] == "rotary":
        heads = hk if case["move"] else hq + hk
        return {"bytes": case["n"] * (2 * heads * d * e + (8 if case["move"] else 4)), "flops": 3.0 * case["n"] * heads * case["part"]}
    if case["op"] == "store":
        n, nb = case["n"], min(case["n"], -(-case["n_rows"] // case["block"]))
        return {"bytes": n * (2 * hk * d * (e + 1) + 1 + 4 * hk + (0 if case["rows"] == "whole" else 4)) + 16 * nb * hk, "flops": 4.0 * n * hk * d}
    if case["op"] == "deviation":
        n, t = case["n"], 2 if case["mode"] == "kv" else 1
        return {"bytes": n * (t * hk * d * (e + 1) + 5 + 4 * hk * (t + (1 if case["alpha"] else 0))) + 4 * t * hk * (n // case["block"] + 1), "flops": 3.0 * n * t * hk * d}
    # on average: picked rows lie anywhere in their contexts, a decode step's at their ends
    length, rows = 0.5 * (case["lo"] + case["hi"]), case["rows"]
    live = case["batch"] - case["idle"]
    seen = length * (1.0 if rows <= 4 else 0.5)
    keys = live * length * (1.0 if rows <= 4 else rows / (rows + 1.0))
    return {"bytes": keys * hk * (2 * d + 8.0 / case["block"]) + case["batch"] * rows * (hq * (2 * d * e + 4) + 4), "flops": 4.0 * d * hq * live * rows * seen}


def exact(case, seed):
    s = prepare(case, seed)
    hq, hk, d = HEADS[case["model"]]
    if case["op"] == "rotary":
        a = _rotary_args(case)
        r, n = a["rotary_dim"], case["n"]
        shift = s["pos"].double() - (s["pos_from"].double() if case["move"] else 0.0)
        turn = torch.polar(torch.full((n, r // 2), a["magnitude"], dtype=torch.float64, device=DEV), shift[:, None] * _exact_frequencies(a))
        out = []
        for x in (s["q"], s["k"]):
            if x is not None:
                y = x.double().clone()
                pair = (y[..., 0:r:2], y[..., 1:r:2]) if a["layout"] == "interleaved" else (y[..., : r // 2], y[..., r // 2: r])
                z = torch.complex(pair[0].contiguous(), pair[1].contiguous()) * turn[:, None]
                pair[0].copy_(z.real)
                pair[1].copy_(z.imag)
                out.append(y)
        return out
    if case["op"] == "store":
        return _exact_store(s)
    if case["op"] == "deviation":
        block = torch.arange(case["n"], device=DEV) // case["block"]
        dev = {x: (s[x + "_fresh"].double() - s[x].double() * s[x + "_scale"].double()[block].unsqueeze(-1)).abs().sum(-1).T for x in ("k", "v")}
        weight = s["alpha"].double() if case["alpha"] else torch.ones_like(dev["v"])
        score = (weight * (dev["v"] + dev["k"] if case["mode"] == "kv" else dev["v"])).sum(0)
        score[s["reused"] == 0] = -math.inf
        return ([dev["k"].contiguous()] if case["mode"] == "kv" else []) + [dev["v"].contiguous(), score]
    out, lse = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV), torch.full(s["lse"].shape, -math.inf, dtype=torch.float64, device=DEV)
    for b, (o, n) in enumerate(zip(s["ctx_off"], s["ctx_len"])):
        mine = slice(s["cu_sel"][b], s["cu_sel"][b + 1])
        seen = torch.arange(n, device=DEV)[None] <= s["pos"][mine, None]
        block = torch.arange(o, o + n, device=DEV) // case["block"]
        for g in range(hk):
            k, v = (s[x][o:o + n, g].double() * s[x + "_scale"].double()[block, g][:, None] for x in ("k", "v"))
            for h in range(g * (hq // hk), (g + 1) * (hq // hk)):
                logit = torch.where(seen, s["q"][mine, h].double() @ k.T, -math.inf)
                lse[mine, h] = torch.logsumexp(logit, 1)
                out[mine, h] = torch.where(seen.any(1, keepdim=True), torch.softmax(logit, 1) @ v, 0.0)
    return [out, lse]


def _exact_frequencies(a):
    r = a["rotary_dim"]
    found = []
    for j in range(r // 2):
        f = a["base"] ** (-2.0 * j / r)
        if a["scaling"] == "ntk":
            f = (a["base"] * a["factor"] ** (r / (r - 2.0))) ** (-2.0 * j / r)
        elif a["scaling"] == "linear":
            f = f / a["factor"]
        elif a["scaling"] == "wavelength":
            wave = 2 * math.pi / f
            if wave > a["original"] / a["low"]:
                f = f / a["factor"]
            elif wave > a["original"] / a["high"]:
                smooth = (a["original"] / wave - a["low"]) / (a["high"] - a["low"])
                f = (1 - smooth) * f / a["factor"] + smooth * f
        elif a["scaling"] == "ramp":
            first, last = (r / 2.0 * math.log(a["original"] / (2 * math.pi * t), a["base"]) for t in (a["high"], a["low"]))
            first, last = max(math.floor(first), 0), min(math.ceil(last), r - 1)
            slow = min(max((j - first) / max(last - first, 0.001), 0.0), 1.0)
            f = f * (1.0 - slow + slow / a["factor"])
        found.append(f)
    return torch.tensor(found, dtype=torch.float64, device=DEV)


def _exact_store(s):
    """Codes are whole steps of scales in 32 bits, so those of int8 have no value apart from that definition; the other outputs do."""
    case = s["case"]
    n_rows, blk, top = case["n_rows"], case["block"], TOP[case["code"]]
    nb = -(-n_rows // blk)
    given = torch.zeros((nb * blk,), dtype=torch.bool, device=DEV)
    given[torch.arange(case["n"], device=DEV) if s["pos"] is None else s["pos"].long()] = True
    inside = torch.arange(nb * blk, device=DEV) < n_rows
    found = {}
    for x in ("k", "v"):
        hk, d = s[x].shape[1:]
        new = torch.zeros((nb * blk, hk, d), dtype=torch.float64, device=DEV)
        new[given] = s[x + "_new"].double()
        mine = new.view(nb, blk, hk, d).abs().amax((1, 3)) / top
        kept = (inside & ~given).view(nb, blk).any(1)
        scale = torch.where(kept[:, None], torch.maximum(s[x + "_scale"].double(), mine), mine)
        found[x + "_scale"] = scale
        if case["code"] == "int8":
            found[x] = None
        else:
            whole = scale.repeat_interleave(blk, 0)[:, :, None]
            held = torch.zeros_like(new)
            held[:n_rows] = s[x].double() * s[x + "_scale"].double().repeat_interleave(blk, 0)[:n_rows, :, None]
            value = torch.where(given[:, None, None], new, held) / whole.clamp_min(1e-300)
            found[x] = _nearest_e4m3(value)[:n_rows].contiguous()
    dev_v = s["dev_v"].double()
    dev_v[:, given[:n_rows]] = 0.0
    return [found["k"], found["v"], found["k_scale"], found["v_scale"], None, dev_v]


def _nearest_e4m3(y):
    """Three bits behind the leading one, exponents from -6 on, at most 448."""
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp_min(2.0 ** -6))) - 3.0)
    return ((y / step).round() * step).clamp(-448.0, 448.0)
