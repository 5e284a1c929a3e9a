"""kvs_attention_kv8, launches of many rows, which widen their contexts to bf16 in the workspace first (bf16, head_dim 128, from 7373
rows on, where the bytes of the copy pay), against attention in 64 bits."""
import numpy as np
import pytest
import torch

import kv8_ref as R
from paper_2503_16525_amd import binding as B

pytestmark = pytest.mark.gpu


def _reference(q, pos, k, v, scale):
    """R.attention for many rows at once: torch float64 on the GPU, a query head at a time."""
    n, hq, d = q.shape
    grp = hq // k.shape[1]
    qd, kd, vd = (torch.from_numpy(x).cuda() for x in (q, k, v))
    p = torch.tensor(pos).cuda().clamp_max(k.shape[0] - 1)
    seen = torch.arange(k.shape[0], device="cuda")[None] <= p[:, None]
    out, mag, lse, dots = np.zeros((n, hq, d)), np.zeros((n, hq, d)), np.full((n, hq), -np.inf), 0.0
    for h in range(hq):
        kh = kd[:, h // grp].contiguous()
        s = scale * (qd[:, h].contiguous() @ kh.T.contiguous())
        dots = max(dots, float((abs(scale) * (qd[:, h].abs() @ kh.abs().T.contiguous())).max()))
        s = torch.where(seen, s, -torch.inf)
        w = torch.where(seen.any(1, keepdim=True), torch.softmax(s, 1), 0.0)
        vh = vd[:, h // grp].contiguous()
        out[:, h], mag[:, h], lse[:, h] = (x.cpu().numpy() for x in (w @ vh, w @ vh.abs(), torch.logsumexp(s, 1)))
    return out, lse, mag, dots, R.largest(v, hq)


def _case(hq, hk, code, block, reqs, seed, scale=1.0, change=None, want_lse=True, stretch=None, widened=True):
    off, ln, cu, pos, at = [], [], [0], [], 0
    for gap, n, p in reqs:
        at += gap
        off.append(at)
        ln.append(n)
        at += n
        pos += [int(x) for x in p]
        cu.append(len(pos))
    rng = np.random.default_rng(seed)
    x = rng.normal(0, 1, (2, at, hk, 128)).astype(np.float32)
    if stretch is not None:
        stretch(x)
    cache = []
    for t in range(2):                                     # whole blocks at once
        nb = -(-at // block)
        pad = np.zeros((nb * block, hk, 128), np.float32)
        pad[:at] = x[t]
        s = np.abs(pad).reshape(nb, block, hk, 128).max((1, 3)) * (np.float32(1) / R.TOP[code])
        codes = R.nearest(x[t] * (np.float32(1) / s).repeat(block, 0)[:at, :, None], code)
        cache += [codes, s]
    if change is not None:
        change(cache, off, ln)
    kh, vh = (np.nan_to_num(R.held(cache[i], cache[i + 1], block, code)) for i in (0, 2))
    q = (torch.randn((len(pos), hq, 128), generator=torch.Generator().manual_seed(seed)) / (128 ** 0.5 * abs(scale))).to(torch.bfloat16)
    ref = R.joined([_reference(q[cu[b]:cu[b + 1]].double().numpy(), pos[cu[b]:cu[b + 1]], kh[off[b]:off[b] + ln[b]], vh[off[b]:off[b] + ln[b]], scale)
                    for b in range(len(ln)) if cu[b + 1] > cu[b]])
    gpu, sh = R.on_gpu(B, cache, block, code), B.make_shape(hq, hk, 128, B.BF16)
    what = f"{hq}x{hk}, {code}/{block}, {len(ln)} requests of {min(ln)} to {max(ln)}, {len(pos)} tokens"
    print(what, flush=True)
    call = (sh, gpu, off, ln, cu, q.cuda(), torch.tensor(pos, dtype=torch.int32).cuda(), scale)
    ws = torch.full((B.kvs_workspace_size("attention_kv8", sh, len(ln), at, len(pos)),), 255, dtype=torch.uint8, device="cuda")
    out, lse = torch.full_like(q, 7.0).cuda(), torch.full((len(pos), hq), 7.0, device="cuda")
    B.kvs_attention_kv8(*call, out, lse if want_lse else None, ws)
    R.check_attention(out.float().cpu().numpy(), lse.cpu().numpy() if want_lse else ref[1], ref, "bf16", max(ln), what, widened)
    assert bool((ws[-hk * 8 - 512 - 256 * hk * min(ln):] != 255).any()) == widened, "whether the copy was made"
    if not widened:
        return call, ref
    # without room for the copy the codes are widened where they are used
    out2, lse2 = torch.full_like(q, 7.0).cuda(), torch.full((len(pos), hq), 7.0, device="cuda")
    B.kvs_attention_kv8(*call, out2, lse2 if want_lse else None, None)
    R.check_attention(out2.float().cpu().numpy(), lse2.cpu().numpy() if want_lse else ref[1], ref, "bf16", max(ln), what + ", without a workspace")
    return call, ref


def _pick(rng, n, k):
    return np.sort(rng.permutation(n)[:k])


@pytest.mark.parametrize("code,block", [("e4m3", 32), ("int8", 16), ("e4m3", 128), ("int8", 64)])
@pytest.mark.parametrize("hq,hk,n,k_sel", [(32, 8, 9000, 3000), (28, 4, 8003, 3100), (32, 4, 12001, 1900), (56, 8, 6001, 2900)])
def test_one_request(hq, hk, n, k_sel, code, block):
    rng = np.random.default_rng(n)
    _case(hq, hk, code, block, [(16 * (n % 5), n, _pick(rng, n, k_sel))], seed=n)


@pytest.mark.parametrize("code", ["e4m3", "int8"])
def test_ragged_batches(code):
    """Contexts of one row and up, whole prompts, rows that see nothing, any order, the same twice; contexts that begin inside 16 rows."""
    rng = np.random.default_rng(1)
    pad = lambda n: -n % 16
    lens = [4300, 1, 17, 5200, 31, 32, 33, 3047]
    reqs, before = [], 0
    for n in lens:
        reqs.append((pad(before), n, _pick(rng, n, max(1, n * 2 // 3))))
        before = n
    _case(32, 8, code, 32, reqs, seed=2)
    _case(32, 8, code, 16, [(0, 6000, rng.integers(-3, 6020, 2500)), (0, 16, []), (0, 4208, rng.permutation(4208)[:2400]), (16, 100, [-1] * 30), (12, 90, [5, 5, 0])], seed=3)
    _case(16, 16, code, 64, [(0, 7000, range(7000))], seed=4, want_lse=False, scale=0.5)
    _case(32, 8, code, 16, [(0, 3000, _pick(rng, 3000, 1500)), (5, 3000, _pick(rng, 3000, 1500))], seed=5, widened=False)


@pytest.mark.parametrize("code", ["e4m3", "int8"])
def test_odd_bytes_and_scales(code):
    """Bytes of every kind outside the context and in blocks of scale 0; scales of K and V far from 1."""
    def change(cache, off, ln):
        first, end = off[0], 5000 + off[0]                  # nobody looks further than position 4999
        for x in (0, 2):
            cache[x][:first] = 0xFF
            cache[x][end:] = 0x7F
            cache[x][first + 320:first + 336] = 0xFF
            cache[x + 1][first // 16 + 20] = 0.0
            cache[x + 1][:first // 16] = np.nan
            cache[x + 1][-(-end // 16):] = np.nan
    rng = np.random.default_rng(5)
    _case(32, 8, code, 16, [(48, 5100, _pick(rng, 5000, 4000))], seed=6, change=change)

    def far(cache, off, ln):
        cache[3][:, ::2] *= np.float32(2.0 ** -100)
        cache[3][3:9, 1::2] *= np.float32(2.0 ** 70)
        cache[1][10:12] *= np.float32(2.0 ** -110)
    _case(32, 8, code, 16, [(0, 5000, _pick(rng, 5000, 4000))], seed=7, change=far)


@pytest.mark.parametrize("code", ["e4m3", "int8"])
def test_large_scores(code):
    """Scores that rise by hundreds behind the first tile, and by thousands later; and ones that fall."""
    def rise(x):
        x[0, 300:330] *= 100
        x[0, 700:710] *= 3000
    rng = np.random.default_rng(8)
    _case(32, 8, code, 32, [(0, 5000, _pick(rng, 5000, 4000))], seed=9, stretch=rise)

    def fall(x):
        x[0, :32] *= 300
    _case(32, 8, code, 32, [(0, 5000, _pick(rng, 5000, 4000))], seed=10, stretch=fall)


def test_broken_blocks_reach_the_rows_that_see_them():
    rng = np.random.default_rng(11)
    pos = _pick(rng, 6000, 4000)
    call, ref = _case(32, 8, "e4m3", 32, [(32, 6000, pos)], seed=12)
    gpu, q = call[1], call[5]
    ws = torch.empty((B.kvs_workspace_size("attention_kv8", call[0], 1, gpu.n_rows, len(pos)),), dtype=torch.uint8, device="cuda")
    for x in (gpu.k_scale, gpu.v_scale):
        was = x[100, 5].clone()
        x[100, 5] = float("nan")
        out = torch.full_like(q, 7.0)
        B.kvs_attention_kv8(*call, out, None, ws)
        got = out.float().cpu().numpy()
        broken = np.zeros((len(pos), 32), bool)
        broken[pos >= 99 * 32, 20:24] = True
        assert np.isnan(got[broken]).all() and np.isfinite(got[~broken]).all()
        assert (np.abs(got[~broken] - ref[0][~broken]) <= 2.0 ** -8 * 4 * ref[2][~broken] + 1e-5).all()
        x[100, 5] = was


def test_replays_from_a_graph():
    rng = np.random.default_rng(13)
    call, _ = _case(28, 4, "int8", 64, [(0, 6000, _pick(rng, 6000, 1500))], seed=14)
    sh, gpu, q = call[0], call[1], call[5]
    ws = [torch.empty((B.kvs_workspace_size("attention_kv8", sh, 1, 6000, 1500),), dtype=torch.uint8, device="cuda") for _ in range(2)]
    outs, lses = [torch.empty_like(q) for _ in range(2)], [torch.empty((1500, 28), device="cuda") for _ in range(2)]
    B.kvs_attention_kv8(*call, outs[0], lses[0], ws[0])
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        B.kvs_attention_kv8(*call, outs[1], lses[1], ws[1])
    for i in range(3):
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(outs[0], outs[1]) and torch.equal(lses[0], lses[1]), i
        q.mul_(-1.5)
        gpu.k_scale.mul_(1.1)
        B.kvs_attention_kv8(*call, outs[0], lses[0], ws[0])
