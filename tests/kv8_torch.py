"""The 8-bit cache and attention over it in torch on the GPU, for tests too large for numpy: codes of normal values, what they stand
for in 64 bits, and attention in 64 bits, a query head at a time."""
import torch

from paper_2503_16525_amd import binding as B

TOP = {"e4m3": 448.0, "int8": 127.0}


def quantise(x, block, code):
    """fp32 [rows, heads, d] -> codes, fp32 scales [blocks, heads]: a cache that stands for nearly x"""
    n = x.shape[0]
    nb = -(-n // block)
    most = torch.zeros((nb * block, x.shape[1]), device=x.device)
    most[:n] = x.abs().amax(-1)
    scale = (most.view(nb, block, -1).amax(1) / TOP[code]).clamp_min(2.0 ** -126)
    y = (x / scale.repeat_interleave(block, 0)[:n, :, None]).clamp(-TOP[code], TOP[code])
    return (y.to(torch.float8_e4m3fn) if code == "e4m3" else y.round().to(torch.int8)), scale


def normal_cache(n_rows, hk, d, block, code, seed, change=None):
    """change(x): x is K, then V, in fp32, in place"""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    out = []
    for t in range(2):
        x = torch.randn((n_rows, hk, d), generator=gen, device="cuda")
        if change is not None:
            change(x, t)
        out += quantise(x, block, code)
    return B.Cache8(out[0], out[2], out[1], out[3], block)


def held(codes, scale, block, lo, n, g):
    """rows lo .. lo + n - 1 of head g in 64 bits"""
    rows = torch.arange(lo, lo + n, device=codes.device)
    return codes[lo:lo + n, g].float().double() * scale[rows // block, g].double()[:, None]


def attention(q, pos, cache, off, ln, cu, scale):
    """-> out, lse, sum of |weight * v| (64 bits, [tokens, query heads, ..]), largest sum of |q k|, largest |v| of each query head"""
    n, hq, d = q.shape
    grp = hq // cache.n_kv_heads
    out, mag = (torch.zeros((n, hq, d), dtype=torch.float64, device="cuda") for _ in range(2))
    lse = torch.full((n, hq), -torch.inf, dtype=torch.float64, device="cuda")
    most, dots = torch.zeros((hq,), dtype=torch.float64, device="cuda"), 0.0
    for b in range(len(ln)):
        a, e = cu[b], cu[b + 1]
        if e == a or ln[b] == 0:
            continue
        seen = torch.arange(ln[b], device="cuda")[None] <= pos[a:e, None].long().clamp_max(ln[b] - 1)
        some = seen.any(1, keepdim=True)
        for h in range(hq):
            g = h // grp
            k, v = (held(c, s, cache.block, off[b], ln[b], g) for c, s in ((cache.k, cache.k_scale), (cache.v, cache.v_scale)))
            qh, kt = q[a:e, h].double().contiguous(), k.T.contiguous()
            s = torch.where(seen, scale * (qh @ kt), -torch.inf)
            dots = max(dots, float(abs(scale) * (qh.abs() @ kt.abs()).max()))
            w = torch.where(some, torch.softmax(s, 1), 0.0)
            out[a:e, h], mag[a:e, h] = w @ v, w @ v.abs()
            lse[a:e, h] = torch.logsumexp(s, 1)
            most[h] = torch.maximum(most[h], v.abs().max())
    return out, lse, mag, dots, most


def off_by(out, want):
    """norm of the difference over the norm"""
    return float((out.double() - want).norm() / want.norm())
