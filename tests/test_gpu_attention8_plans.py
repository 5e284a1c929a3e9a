"""kvs_attention_kv8 where its key ranges are cut and its requests are laid out in one of several ways: few and many pieces, few and
many blocks of rows, batches whose requests differ, hold no rows or no keys, against attention in 64 bits."""
import numpy as np
import pytest
import torch

import kv8_ref as R
from paper_2503_16525_amd import binding as B
from test_gpu_attention8_wide import _reference

pytestmark = pytest.mark.gpu


def _case(hq, hk, d, dtype, code, block, reqs, seed, fractions=(1.0,)):
    """reqs: (rows of the cache before the context, its length, positions); fractions: of the workspace asked for."""
    off, ln, cu, pos, at = [], [], [0], [], 0
    for gap, n, p in reqs:
        at += gap
        off.append(at)
        ln.append(n)
        at += n
        pos += [int(x) for x in p]
        cu.append(len(pos))
    at += 3
    cache = R.make(at, hk, d, block, code, seed) if at < 4000 else _levels(at, hk, d, block, code, seed)
    kh, vh = R.held(cache[0], cache[1], block, code), R.held(cache[2], cache[3], block, code)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    q = (torch.randn((len(pos), hq, d), generator=torch.Generator().manual_seed(seed)) / d ** 0.5).to(dt)
    parts = []
    for b in range(len(ln)):
        n = cu[b + 1] - cu[b]
        if n and ln[b]:
            parts.append(_reference(q[cu[b]:cu[b + 1]].double().numpy(), pos[cu[b]:cu[b + 1]], kh[off[b]:off[b] + ln[b]], vh[off[b]:off[b] + ln[b]], 1.0))
        elif n:
            parts.append((np.zeros((n, hq, d)), np.full((n, hq), -np.inf), np.zeros((n, hq, d)), 0.0, np.zeros(hq)))
    ref = R.joined(parts)
    gpu, sh = R.on_gpu(B, cache, block, code), B.make_shape(hq, hk, d, B.BF16 if dtype == "bf16" else B.F32)
    sel = torch.tensor(pos, dtype=torch.int32).cuda()
    size = B.kvs_workspace_size("attention_kv8", sh, len(ln), at, len(pos))
    for f in fractions:
        what = f"{hq}x{hk}x{d} {dtype}, {code}/{block}, {len(ln)} requests of {min(ln)} to {max(ln)}, {len(pos)} tokens, {f} of the workspace"
        print(what, flush=True)
        ws = torch.full((int(size * f) // 256 * 256,), 255, dtype=torch.uint8, device="cuda") if f else None
        out, lse = torch.full_like(q, 7.0).cuda(), torch.full((len(pos), hq), 7.0, device="cuda")
        B.kvs_attention_kv8(sh, gpu, off, ln, cu, q.cuda(), sel, 1.0, out, lse, ws)
        R.check_attention(out.float().cpu().numpy(), lse.cpu().numpy(), ref, dtype, max(ln), what)


def _levels(n, hk, d, block, code, seed):
    """As kv8_ref.make, whole blocks at once."""
    rng = np.random.default_rng(seed)
    cache, nb = [], -(-n // block)
    for _ in range(2):
        x = (rng.normal(0, 1, (n, hk, d)) * np.exp(rng.normal(0, 0.5, (nb, hk))).repeat(block, 0)[:n, :, None]).astype(np.float32)
        pad = np.zeros((nb * block, hk, d), np.float32)
        pad[:n] = x
        s = np.abs(pad).reshape(nb, block, hk, d).max((1, 3)) * (np.float32(1) / R.TOP[code])
        cache += [R.nearest(x * (np.float32(1) / s).repeat(block, 0)[:n, :, None], code), s]
    return cache


def _pick(rng, n, k):
    return np.sort(rng.permutation(n)[:k])


HEADS = [(32, 8, 128, "bf16"), (28, 4, 64, "bf16"), (4, 4, 64, "f32"), (12, 3, 128, "f32")]


@pytest.mark.parametrize("code", ["e4m3", "int8"])
@pytest.mark.parametrize("hq,hk,d,dtype", HEADS)
@pytest.mark.parametrize("n,k", [(257, 3), (1500, 40), (2999, 9), (3500, 150), (9001, 1), (12000, 33)])
def test_one_context(hq, hk, d, dtype, code, n, k):
    rng = np.random.default_rng(n)
    pos = _pick(rng, n, k)
    pos[-1] = n - 1
    _case(hq, hk, d, dtype, code, 32, [(n % 23, n, pos)], n, (1.0, 0.3, 0.0))


@pytest.mark.parametrize("code", ["e4m3", "int8"])
@pytest.mark.parametrize("hq,hk,d,dtype", HEADS)
def test_batches(hq, hk, d, dtype, code):
    """Requests of like sizes, of very different ones, without rows, without keys, with places that hold no token."""
    rng = np.random.default_rng(3)
    _case(hq, hk, d, dtype, code, 16, [(1, n, _pick(rng, n, n // 40)) for n in (700, 640, 1000, 930)], 4, (1.0, 0.1))
    _case(hq, hk, d, dtype, code, 64, [(0, 1500, _pick(rng, 1500, 60)), (5, 40, []), (2, 0, [0, -1, 5]), (0, 17, [16, 16, -1]), (9, 900, [2000, 3]), (0, 1, [0])], 5, (1.0, 0.2))
    _case(hq, hk, d, dtype, code, 128, [(0, n, [n - 1]) for n in (1400, 3, 1100, 1, 64, 512, 33, 900)], 6)
    _case(hq, hk, d, dtype, code, 32, [(0, 0, [3, -1]), (0, 0, [0])], 7)


def test_a_cache_of_no_rows():
    sh = B.make_shape(8, 2, 128, B.BF16)
    cache = B.Cache8.empty(sh, 0, 32)
    q = torch.randn((3, 8, 128)).to(torch.bfloat16).cuda()
    out, lse = torch.full_like(q, 7.0), torch.full((3, 8), 7.0).cuda()
    B.kvs_attention_kv8(sh, cache, [0, 0], [0, 0], [0, 2, 3], q, torch.tensor([0, -1, 5], dtype=torch.int32).cuda(), 1.0, out, lse, None)
    assert not out.any() and torch.isneginf(lse).all()
