"""kvs_rotary against the rotation in 64 bits: layouts, parts of the head, scalings, moves, strides, in place."""
import math

import numpy as np
import pytest
import torch

from paper_2503_16525_amd import binding as B

pytestmark = pytest.mark.gpu

SCALINGS = {"plain": {}, "linear": dict(factor=4.0), "ntk": dict(factor=4.0), "ramp": dict(factor=8.0, original=4096, low=1.0, high=32.0),
            "wavelength": dict(factor=8.0, original=8192, low=1.0, high=4.0)}


def _frequencies(r, scaling, base, factor=1.0, original=0, low=1.0, high=4.0):
    f = []
    for j in range(r // 2):
        x = base ** (-2.0 * j / r)
        if scaling == "linear":
            x /= factor
        elif scaling == "ntk":
            x = (base * factor ** (r / (r - 2.0))) ** (-2.0 * j / r)
        elif scaling == "wavelength":
            turns = original * x / (2 * math.pi)
            w = min(max((turns - low) / (high - low), 0.0), 1.0)
            x = w * x + (1 - w) * x / factor
        elif scaling == "ramp":
            at = [r * math.log(original / (t * 2 * math.pi)) / (2 * math.log(base)) for t in (high, low)]
            lo, hi = max(math.floor(at[0]), 0), min(math.ceil(at[1]), r - 1)
            w = min(max((j - lo) / max(hi - lo, 0.001), 0.0), 1.0)
            x = (1 - w) * x + w * x / factor
        f.append(x)
    return np.array(f)


def _turned(x, shift, f, layout, magnitude):
    """float64 [n, heads, d] turned, and |u| + |v| of each channel's pair"""
    r = 2 * len(f)
    c, s = np.cos(shift[:, None] * f)[:, None] * magnitude, np.sin(shift[:, None] * f)[:, None] * magnitude
    iu, iv = (np.arange(0, r, 2), np.arange(1, r, 2)) if layout == "interleaved" else (np.arange(r // 2), np.arange(r // 2, r))
    y, size = x.copy(), np.zeros_like(x)
    u, v = x[..., iu], x[..., iv]
    y[..., iu], y[..., iv] = u * c - v * s, v * c + u * s
    size[..., iu] = size[..., iv] = abs(magnitude) * (np.abs(u) + np.abs(v))
    return y, size


def _check(got, x, shift, f, layout, magnitude, what):
    """A store's rounding (half a step), and for each of the two products of a turned channel: an angle off by 2^-26 of a turn
    (1e-7, 1.6 roundings), sine, cosine and magnitude by 4 roundings, product and sum by 2."""
    want, size = _turned(x.double().cpu().numpy(), shift, f, layout, magnitude)
    half = torch.finfo(got.dtype).eps / 2
    tol = half * np.abs(want) + 8 * 2.0 ** -24 * size
    err = np.abs(got.double().cpu().numpy() - want)
    assert (err <= tol).all(), f"{what}: off by {err.max()}, bound there {tol[np.unravel_index((err - tol).argmax(), err.shape)]}"


@pytest.mark.parametrize("scaling", SCALINGS)
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("hq,hk,d,dtype", [(28, 4, 128, torch.bfloat16), (4, 4, 64, torch.float32), (3, 1, 64, torch.bfloat16), (5, 5, 128, torch.float32)])
def test_fresh_rows(hq, hk, d, dtype, layout, scaling):
    sh = B.make_shape(hq, hk, d, B.BF16 if dtype is torch.bfloat16 else B.F32)
    args = dict(scaling=scaling, base=10000.0, **SCALINGS[scaling])
    for n, part, first in ((1, d, 123456), (17, d // 2, 0), (600, d, 5000), (33, 48, 100), (3, 2, 7), (2, 20, 999983), (1, d - 2, 0)):
        if scaling == "ntk" and part == 2:
            continue
        gen = torch.Generator().manual_seed(n + part)
        q, k = (torch.randn((n, h, d), generator=gen).to(dtype).cuda() for h in (hq, hk))
        pos = torch.arange(first, first + n, dtype=torch.int32).cuda()
        qo, ko = torch.full_like(q, 7.0), torch.full_like(k, 7.0)
        B.kvs_rotary(sh, B.rotary_spec(part, layout, magnitude=1.25, **args), pos, None, q, k, qo, ko)
        f = _frequencies(part, **args)
        for got, x, what in ((qo, q, "q"), (ko, k, "k")):
            _check(got, x, pos.double().cpu().numpy(), f, layout, 1.25, f"{what}, {n} rows, {part} of {d} channels, {layout}, {scaling}")


@pytest.mark.parametrize("layout,part", [("half", 128), ("interleaved", 64), ("half", 20)])
def test_moved_keys_and_strides(layout, part):
    """Keys out of a fused buffer, from one position to another, far apart both ways; then back again, in place."""
    hq, hk, d, n = 6, 2, 128, 1500
    sh = B.make_shape(hq, hk, d, B.BF16)
    gen = torch.Generator().manual_seed(part)
    buf = torch.randn((n, hq + 2 * hk + 1, d), generator=gen).to(torch.bfloat16).cuda()
    was = buf.clone()
    k = buf[:, hq:hq + hk]
    a, b = (torch.randint(-(1 << 20), 1 << 20, (n,), generator=gen, dtype=torch.int32).cuda() for _ in range(2))
    out = torch.full((n + 2, hk + 1, d), 7.0, dtype=torch.bfloat16, device="cuda")
    spec = B.rotary_spec(part, layout)
    B.kvs_rotary(sh, spec, a, b, None, k, None, out[1:-1, :hk])
    f = _frequencies(part, "plain", 10000.0)
    _check(out[1:-1, :hk], k, (a.double() - b.double()).cpu().numpy(), f, layout, 1.0, "moved")
    assert (out[0] == 7).all() and (out[-1] == 7).all() and (out[:, hk] == 7).all() and torch.equal(buf, was)
    # in place, and nothing beside the keys changes
    B.kvs_rotary(sh, spec, a, b, None, k, None, k)
    assert torch.equal(buf[:, hq:hq + hk], out[1:-1, :hk])
    assert torch.equal(buf[:, :hq], was[:, :hq]) and torch.equal(buf[:, hq + hk:], was[:, hq + hk:])


def test_scores_go_by_the_difference_of_positions():
    """q at p and k at p - 5: the same dot products at any p, which is what lets a reused key move; the moved key gives them too."""
    d, n = 64, 40
    sh = B.make_shape(2, 2, d, B.F32)
    spec = B.rotary_spec(d, "half", "wavelength", 500000.0, 8.0, 8192, 1.0, 4.0)
    gen = torch.Generator().manual_seed(1)
    q, k = (torch.randn((1, 2, d), generator=gen).expand(n, -1, -1).contiguous().cuda() for _ in range(2))
    pos = (torch.arange(n, dtype=torch.int32) * 3001 + 5).cuda()
    qo, ko, km = (torch.empty_like(q) for _ in range(3))
    B.kvs_rotary(sh, spec, pos, None, q, None, qo, None)
    B.kvs_rotary(sh, spec, pos - 5, None, None, k, None, ko)
    first = ko[:1].expand(n, -1, -1).contiguous()
    B.kvs_rotary(sh, spec, pos - 5, torch.zeros_like(pos), None, first, None, km)
    # 64 products of numbers below 5, each channel off by 10 roundings (20 after two turns)
    bound = 64 * 25 * 2 * 20 * 2.0 ** -24
    for keys in (ko, km):
        dots = (qo.double() * keys.double()).sum(-1)
        assert float((dots - dots[0]).abs().max()) <= bound


def test_streams_capture_and_device_refusal():
    sh = B.make_shape(4, 4, 64, B.F32)
    spec = B.rotary_spec(64)
    q = torch.randn((50, 4, 64)).cuda()
    pos = torch.arange(50, dtype=torch.int32).cuda()
    want, got = torch.empty_like(q), torch.empty_like(q)
    B.kvs_rotary(sh, spec, pos, None, q, None, want, None)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        B.kvs_rotary(sh, spec, pos, None, q, None, got, None)
    for i in range(3):
        q.copy_(torch.randn((50, 4, 64)))
        B.kvs_rotary(sh, spec, pos, None, q, None, want, None)
        got.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(got, want), i
    with pytest.raises(TypeError):
        B.kvs_rotary(sh, spec, pos, None, q.cpu(), None, got, None)
    with pytest.raises(ValueError):
        B.kvs_rotary(sh, spec, pos[:49], None, q, None, got, None)
    with pytest.raises(TypeError):
        B.kvs_rotary(sh, spec, pos, None, q.transpose(1, 2).contiguous().transpose(1, 2), None, got, None)
