"""The 8-bit cache in plain numpy, for the tests: codes and their values, the store as its definition reads (fp32 where the
definition is), attention and deviation in 64 bits on what a cache stands for."""
import numpy as np
import torch

TOP = {"e4m3": np.float32(448.0), "int8": np.float32(127.0)}
TYPES = {"e4m3": torch.float8_e4m3fn, "int8": torch.int8}


def _e4m3_values():
    c = np.arange(256)
    sign, e, m = np.where(c & 0x80, -1.0, 1.0), (c >> 3) & 15, c & 7
    v = np.where(e == 0, m / 8.0 * 2.0 ** -6, (1.0 + m / 8.0) * 2.0 ** (e - 7.0)) * sign
    v[[0x7F, 0xFF]] = np.nan
    return v


E4M3 = _e4m3_values()


def values(codes, code):
    """uint8 bytes -> float64"""
    return E4M3[codes] if code == "e4m3" else codes.view(np.int8).astype(np.float64)


def nearest(y, code):
    """fp32 numbers -> the bytes of the nearest codes, ties to even, at most the largest"""
    y = np.clip(np.asarray(y, np.float64), -float(TOP[code]), float(TOP[code]))
    if code == "int8":
        return np.rint(y).astype(np.int8).view(np.uint8)
    a = np.abs(y)
    e = np.floor(np.log2(np.maximum(a, 2.0 ** -6)))
    step = 2.0 ** (e - 3)
    a = np.rint(a / step) * step                          # may reach the next power of two, which is a code too
    e = np.floor(np.log2(np.maximum(a, 2.0 ** -6)))
    m = np.rint(a / 2.0 ** (e - 3)).astype(np.int64)      # 8 .. 15, or below 8 under 2^-6
    c = np.where(m >= 8, ((e.astype(np.int64) + 7) << 3) | (m & 7), m)
    return (c | np.where(np.signbit(y), 0x80, 0)).astype(np.uint8)


def store(codes, scale, new, pos, block, code):
    """One tensor of kvs_store_kv8, in place: codes uint8 [rows, heads, d], scale fp32, new fp32 [n, heads, d], pos a list of rows."""
    n_rows, hk, _ = codes.shape
    takes = {}
    for s, p in enumerate(pos):
        if 0 <= p < n_rows:
            takes[int(p)] = s                             # the last of equal entries
    for blk in sorted({p // block for p in takes}):
        rows = range(blk * block, min((blk + 1) * block, n_rows))
        taken = [r for r in rows if r in takes]
        kept = [r for r in rows if r not in takes]
        for g in range(hk):
            x = new[[takes[r] for r in taken], g]
            old = scale[blk, g]
            with np.errstate(all="ignore"):
                most = np.float32(np.abs(x).max()) if x.size else np.float32(0)
                if not np.isfinite(x).all() or (kept and np.isnan(old)):
                    scale[blk, g] = np.nan
                    codes[taken, g] = 0
                    continue
                need = max(most * (np.float32(1) / TOP[code]), np.float32(2.0 ** -126)) if most > 0 else np.float32(0)
                now = max(need, old) if kept else need
                inv = np.float32(1) / now if now > 0 else np.float32(0)
                codes[taken, g] = nearest(x * inv, code)
                if kept and now > 0 and now != old:
                    held = codes[kept, g].copy()
                    if code == "e4m3":
                        held = np.where((held & 0x7F) == 0x7F, held - 1, held).astype(np.uint8)
                    codes[kept, g] = nearest(values(held, code).astype(np.float32) * (old / now), code)
                scale[blk, g] = now


def held(codes, scale, block, code):
    """What a cache stands for, in 64 bits."""
    blk = np.arange(codes.shape[0]) // block
    s = scale.astype(np.float64)[blk][:, :, None]
    return np.where(s == 0, 0.0, values(codes, code) * s)


def attention(q, pos, k, v, scale):
    """q [n, hq, d], pos [n] (negative: sees nothing), k, v [len, hk, d] in 64 bits
    -> out, lse, sum of |weight * v|, largest sum of |q k|, largest |v| of each query head"""
    n, hq, d = q.shape
    ln, hk, _ = k.shape
    grp = hq // hk
    out, lse, mag = np.zeros((n, hq, d)), np.full((n, hq), -np.inf), np.zeros((n, hq, d))
    dots = 0.0
    for i in range(n):
        p = min(int(pos[i]), ln - 1)
        if p < 0:
            continue
        for g in range(hk):
            qq = q[i, g * grp:(g + 1) * grp]
            s = scale * (qq @ k[: p + 1, g].T)
            dots = max(dots, float(abs(scale) * (np.abs(qq) @ np.abs(k[: p + 1, g]).T).max()))
            m = s.max(1, keepdims=True)
            w = np.exp(s - m)
            t = w.sum(1, keepdims=True)
            out[i, g * grp:(g + 1) * grp] = w @ v[: p + 1, g] / t
            mag[i, g * grp:(g + 1) * grp] = w @ np.abs(v[: p + 1, g]) / t
            lse[i, g * grp:(g + 1) * grp] = (m + np.log(t))[:, 0]
    return out, lse, mag, dots, largest(v, hq)


def largest(v, hq):
    return np.abs(v).max((0, 2), initial=0.0).repeat(hq // v.shape[1])


def joined(parts):
    """The results of several requests' attention as one's."""
    return [np.concatenate([p[i] for p in parts]) for i in range(3)] + [max(p[3] for p in parts), np.max([p[4] for p in parts], 0)]


def check_attention(out, lse, ref, dtype, longest, what, widened=False):
    """bf16: a weight's rounding, 2^-8 of it, moves the output by at most that share of sum |weight| |v - out| <= 2 mag; the store
    rounds once more.  fp32 everywhere: a score's error is at most (d + 4) roundings of its sum of |q k| (`dots`), its weight's
    that plus a few units; a sum over n keys is off by at most n roundings of its magnitude, numerator and denominator.
    Weights of nothing: the row's largest enters the second product as at least 2^-31 of V's scale (the exponents' reference lies at
    most 31 above the first tile's maximum), bf16 ends at 2^-126, so with scales from 2^-14 up a weight below 2^-126+31+14 of
    the largest may become 0; n of them move the output by less than n 2^-80 max |v|.
    widened: V is rounded to bf16 too, 2^-8 of each |v|, and the exponents' reference lies at most 61 above the first tile's maximum:
    2^-126+61 of the largest; and a product of a weight and a V below 2^-126 may become 0, which against a sum of weights of at least
    2^-61 is 2^-65 of the output for each key."""
    want, want_lse, mag, dots, most = ref
    out, lse = out.astype(np.float64), lse.astype(np.float64)
    assert np.isfinite(out).all(), f"{what}: not finite"
    weight = (132 * dots + 64) * 2.0 ** -24
    tol = mag * 2 * (weight + longest * 2.0 ** -24) + 1e-30
    if dtype == "bf16":
        tol = tol + 2.0 ** -8 * ((3 if widened else 2) * mag + np.abs(want)) + longest * 2.0 ** (-64 if widened else -80) * most[None, :, None]
        tol = tol + (longest * 2.0 ** -65 if widened else 0.0)
    else:
        tol = tol + 2.0 ** -23 * np.abs(want)
    over = np.abs(out - want) - tol
    assert (over <= 0).all(), f"{what}: off by {np.abs(out - want).max()}, {over.max()} above the bound, at {np.unravel_index(over.argmax(), over.shape)}"
    empty = np.isneginf(want_lse)
    assert (np.isneginf(lse) == empty).all(), f"{what}: empty rows"
    err = np.abs(np.where(empty, 0, lse) - np.where(empty, 0, want_lse))
    bound = weight + longest * 2.0 ** -24 + 2.0 ** -22 * np.abs(np.where(empty, 0, want_lse))
    assert (err <= bound).all(), f"{what}: log-sum-exp off by {err.max()}"


def make(n_rows, hk, d, block, code, seed, spread=1.0):
    """codes, scales (uint8, fp32) of a cache of n_rows rows of normal values, each block at a level of its own"""
    rng = np.random.default_rng(seed)
    nb = -(-n_rows // block)
    out = []
    for _ in range(2):
        level = np.exp(rng.normal(0, 0.5, (nb, hk))).repeat(block, 0)[:n_rows, :, None]
        x = (rng.normal(0, spread, (n_rows, hk, d)) * level).astype(np.float32)
        codes, scale = np.zeros((n_rows, hk, d), np.uint8), np.zeros((nb, hk), np.float32)
        store(codes, scale, x, range(n_rows), block, code)
        out += [codes, scale]
    return out


def on_gpu(B, cache, block, code):
    kc, ks, vc, vs = cache
    dt = TYPES[code]
    k, v = (torch.from_numpy(c.copy()).cuda().view(dt) for c in (kc, vc))
    return B.Cache8(k, v, torch.from_numpy(ks.copy()).cuda(), torch.from_numpy(vs.copy()).cuda(), block)
