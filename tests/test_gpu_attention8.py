"""kvs_attention_kv8 against attention in 64 bits on what the cache stands for."""
import numpy as np
import pytest
import torch

import kv8_ref as R
from paper_2503_16525_amd import binding as B

pytestmark = pytest.mark.gpu

SHAPES = [(28, 4, 128), (32, 8, 128), (7, 1, 128), (40, 1, 128), (6, 6, 64), (4, 4, 128), (64, 2, 64)]


def _attend(sh, gpu, off, ln, cu, q, pos, scale, want_ws=True, ws_bytes=None):
    n = q.shape[0]
    out, lse = torch.full_like(q, 7.0), torch.full((n, sh.n_q_heads), 7.0, device="cuda")
    size = ws_bytes if ws_bytes is not None else B.kvs_workspace_size("attention_kv8", sh, len(ln), gpu.n_rows, n) if want_ws else 0
    ws = torch.full((size,), 255, dtype=torch.uint8, device="cuda") if size else None
    B.kvs_attention_kv8(sh, gpu, off, ln, cu, q, pos, scale, out, lse, ws)
    return out.float().cpu().numpy(), lse.cpu().numpy()


def _case(hq, hk, d, dtype, code, block, reqs, scale=1.0, seed=0, slack=0, what=""):
    """reqs: (rows before the context, context length, positions) one after the other."""
    off, ln, cu, pos, at = [], [], [0], [], 0
    for gap, n, p in reqs:
        at += gap
        off.append(at)
        ln.append(n)
        at += n
        pos += list(p)
        cu.append(len(pos))
    n_rows = at + slack
    cache = R.make(max(n_rows, 1), hk, d, block, code, seed)
    gpu = R.on_gpu(B, cache, block, code)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    q = (torch.randn((len(pos), hq, d), generator=torch.Generator().manual_seed(seed)) / (d ** 0.5 * abs(scale) if scale else 1)).to(dt)
    sh = B.make_shape(hq, hk, d, B.BF16 if dtype == "bf16" else B.F32)
    kh, vh = R.held(cache[0], cache[1], block, code), R.held(cache[2], cache[3], block, code)
    parts = [R.attention(q[cu[b]:cu[b + 1]].double().numpy(), pos[cu[b]:cu[b + 1]], kh[off[b]:off[b] + ln[b]], vh[off[b]:off[b] + ln[b]], scale) for b in range(len(ln))]
    ref = R.joined(parts)
    for want_ws in (True, False):
        name = f"{what} {hq}x{hk}x{d} {dtype} {code}/{block}, {len(ln)} requests of {min(ln)} to {max(ln)}, {len(pos)} tokens, workspace {want_ws}"
        print(name, flush=True)
        out, lse = _attend(sh, gpu, off, ln, cu, q.cuda(), torch.tensor(pos, dtype=torch.int32).cuda(), scale, want_ws)
        R.check_attention(out, lse, ref, dtype, max(max(ln), 1), name)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("code", ["e4m3", "int8"])
@pytest.mark.parametrize("hq,hk,d", SHAPES)
def test_single_tokens(hq, hk, d, code, dtype):
    """A decode step: contexts of one row and up, beginning anywhere in a block, the last one at the cache's end."""
    lens = [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 100, 129, 500]
    reqs = [((3 * i) % 7, n, [n - 1]) for i, n in enumerate(lens)]
    _case(hq, hk, d, dtype, code, 16 if hq % 3 else 32, reqs, seed=hq, what="single tokens")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("block,code", [(16, "int8"), (32, "e4m3"), (64, "int8"), (128, "e4m3")])
def test_long_single_tokens_in_pieces(block, code, dtype):
    _case(8, 2, 128, dtype, code, block, [(5, 3001, [3000])], seed=block, what="long")
    _case(8, 2, 128, dtype, code, block, [(0, 2100, [2099]), (1, 40, [39]), (block, 1500, [7, 1499])], seed=block + 1, slack=9, what="ragged")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hq,hk,d,code", [(28, 4, 128, "e4m3"), (8, 8, 64, "int8"), (32, 8, 128, "int8"), (3, 1, 64, "e4m3")])
def test_selected_tokens(hq, hk, d, code, dtype):
    rng = np.random.default_rng(hq)
    pick = lambda n, k: np.sort(rng.permutation(n)[:k]).tolist()
    _case(hq, hk, d, dtype, code, 32, [(0, 700, pick(700, 90))], seed=1, what="one request")
    _case(hq, hk, d, dtype, code, 16, [(3, 260, pick(260, 33)), (0, 1, [0]), (20, 0, []), (1, 90, pick(90, 1)), (0, 333, pick(333, 100))], seed=2, what="ragged")
    # any order, the same twice, none, past the context
    _case(hq, hk, d, dtype, code, 64, [(0, 300, [299, 0, 5, 5, 299, -1, 77, 100000, -1000]), (9, 50, [-1, -1]), (0, 0, [0, -1, 3])], seed=3, what="any order")


def test_every_token_of_a_prompt():
    _case(4, 2, 128, "bf16", "e4m3", 32, [(0, 400, range(400))], seed=5, what="whole prompt")


@pytest.mark.parametrize("scale", [0.125, -0.7, 0.0])
def test_scales_of_the_scores(scale):
    _case(4, 4, 64, "f32", "int8", 16, [(2, 130, [0, 64, 129])], scale=scale, seed=7, what=f"scale {scale}")
    _case(4, 4, 64, "bf16", "e4m3", 16, [(2, 130, [0, 64, 129])], scale=scale, seed=8, what=f"scale {scale}")


def test_more_requests_than_a_launch_describes():
    rng = np.random.default_rng(0)
    lens = rng.integers(1, 90, 150).tolist()
    _case(8, 2, 64, "bf16", "int8", 16, [(i % 3, int(n), [int(n) - 1]) for i, n in enumerate(lens)], seed=9, what="150 requests")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("code", ["e4m3", "int8"])
def test_what_a_row_does_not_see_does_not_reach_it(code, dtype):
    """Bytes of every kind behind the context, before it, in blocks of scale 0 and behind a row's own position; broken blocks
    reach the rows that see them, with their head, and no other."""
    hq, hk, d, block, n = 4, 2, 128, 16, 100
    cache = R.make(n + 60, hk, d, block, code, 11)
    first, ctx = 37, 80
    for x in (0, 2):                                        # codes: NaN ones, outside the context
        cache[x][:first] = 0xFF
        cache[x][first + ctx:] = 0x7F
        cache[x][64:80] = 0xFF                              # a block that holds nothing
        cache[x + 1][4] = 0.0
        cache[x + 1][:2] = np.nan
        cache[x + 1][8:] = np.nan
    # the context is rows 37 .. 116: blocks 2 .. 7, of which the first begins before it
    gpu = R.on_gpu(B, cache, block, code)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    pos = [0, 5, 10, 11, 26, 27, 42, 43, 50, 78, 79]
    q = (torch.randn((len(pos), hq, d), generator=torch.Generator().manual_seed(3)) / d ** 0.5).to(dt)
    sh = B.make_shape(hq, hk, d, B.BF16 if dtype == "bf16" else B.F32)
    p = torch.tensor(pos, dtype=torch.int32).cuda()
    kh, vh = (np.nan_to_num(R.held(cache[x], cache[x + 1], block, code)) for x in (0, 2))
    ref = R.attention(q.double().numpy(), pos, kh[first:first + ctx], vh[first:first + ctx], 1.0)
    for want_ws in (True, False):
        out, lse = _attend(sh, gpu, [first], [ctx], [0, len(pos)], q.cuda(), p, 1.0, want_ws)
        R.check_attention(out, lse, ref, dtype, ctx, f"odd bytes, {code} {dtype}")
    # block 5 (rows 80 .. 95, positions 43 .. 58) of head 1 breaks
    for x in (gpu.k_scale, gpu.v_scale):
        was = x[5, 1].clone()
        x[5, 1] = float("nan")
        out, _ = _attend(sh, gpu, [first], [ctx], [0, len(pos)], q.cuda(), p, 1.0)
        broken = np.zeros((len(pos), hq), bool)
        broken[[i for i, y in enumerate(pos) if y >= 43], 2:] = True
        assert np.isnan(out[broken]).all()
        assert np.isfinite(out[~broken]).all()
        want, got = ref[0][~broken], out[~broken]
        assert (np.abs(got - want) <= 2.0 ** -8 * (3 * ref[2][~broken]) + 1e-5).all()
        x[5, 1] = was


def test_large_scores_and_falling_ones():
    """Scores that rise and fall by hundreds from tile to tile, and rows that one key dominates."""
    hq, hk, d, block, n = 2, 1, 64, 16, 700
    cache = R.make(n, hk, d, block, "int8", 13)
    cache[1][::3] *= 60
    gpu = R.on_gpu(B, cache, block, "int8")
    pos = [0, 15, 16, 300, 699]
    q = torch.randn((len(pos), hq, d), generator=torch.Generator().manual_seed(4))
    kh, vh = (R.held(cache[x], cache[x + 1], block, "int8") for x in (0, 2))
    for dtype, dt in (("f32", torch.float32), ("bf16", torch.bfloat16)):
        qq = q.to(dt)
        ref = R.attention(qq.double().numpy(), pos, kh, vh, 1.0)
        out, lse = _attend(B.make_shape(hq, hk, d, B.BF16 if dtype == "bf16" else B.F32), gpu, [0], [n], [0, 5], qq.cuda(), torch.tensor(pos, dtype=torch.int32).cuda(), 1.0)
        R.check_attention(out, lse, ref, dtype, n, f"large scores, {dtype}")


def test_any_workspace_will_do():
    """From none to what is asked for, on a launch that is cut: the same within the bounds."""
    hq, hk, d, block, n = 4, 1, 128, 32, 5000
    cache = R.make(n, hk, d, block, "e4m3", 17)
    gpu = R.on_gpu(B, cache, block, "e4m3")
    sh = B.make_shape(hq, hk, d, B.BF16)
    q = (torch.randn((3, hq, d), generator=torch.Generator().manual_seed(5)) / d ** 0.5).to(torch.bfloat16)
    pos = [10, 4000, 4999]
    kh, vh = (R.held(cache[x], cache[x + 1], block, "e4m3") for x in (0, 2))
    ref = R.attention(q.double().numpy(), pos, kh, vh, 1.0)
    full = B.kvs_workspace_size("attention_kv8", sh, 1, n, 3)
    for size in (0, 256, 20000, 60001, full // 2, full):
        out, lse = _attend(sh, gpu, [0], [n], [0, 3], q.cuda(), torch.tensor(pos, dtype=torch.int32).cuda(), 1.0, ws_bytes=size)
        R.check_attention(out, lse, ref, "bf16", n, f"workspace of {size}")


def test_replays_from_a_graph():
    hq, hk, d, block, n = 8, 2, 128, 32, 3000
    gpu = R.on_gpu(B, R.make(n, hk, d, block, "e4m3", 19), block, "e4m3")
    sh = B.make_shape(hq, hk, d, B.BF16)
    q = (torch.randn((2, hq, d)) / d ** 0.5).to(torch.bfloat16).cuda()
    pos = torch.tensor([1999, 999], dtype=torch.int32).cuda()
    args = ([0, 2000], [2000, 1000], [0, 1, 2], q, pos, 1.0)
    ws = [torch.empty((B.kvs_workspace_size("attention_kv8", sh, 2, n, 2),), dtype=torch.uint8, device="cuda") for _ in range(2)]
    outs, lses = [torch.empty_like(q) for _ in range(2)], [torch.empty((2, hq), device="cuda") for _ in range(2)]
    B.kvs_attention_kv8(sh, gpu, *args, outs[0], lses[0], ws[0])
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        B.kvs_attention_kv8(sh, gpu, *args, outs[1], lses[1], ws[1])
    for i in range(3):
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(outs[0], outs[1]) and torch.equal(lses[0], lses[1]), i
        q.mul_(-1.25)
        pos.sub_(100)
        B.kvs_attention_kv8(sh, gpu, *args, outs[0], lses[0], ws[0])
