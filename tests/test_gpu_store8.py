"""kvs_store_kv8 against its definition in plain numpy, bit for bit: codes, scales, what is kept and what is rounded again."""
import numpy as np
import pytest
import torch

import kv8_ref as R
from paper_2503_16525_amd import binding as B

pytestmark = pytest.mark.gpu

HEADS = [(4, 64, torch.float32), (8, 128, torch.bfloat16), (1, 128, torch.float32), (3, 64, torch.bfloat16)]


def _new(n, hk, d, dtype, seed, spread=1.0):
    gen = torch.Generator().manual_seed(seed)
    x = torch.randn((n, hk, d), generator=gen) * torch.exp(torch.randn((n, hk, 1), generator=gen)) * spread
    return x.to(dtype)


def _same(cache, kc, ks, vc, vs, what):
    for got, want, name in ((cache.k_scale, ks, "K scales"), (cache.v_scale, vs, "V scales")):
        np.testing.assert_array_equal(got.cpu().numpy(), want, err_msg=f"{what}: {name}")
    for got, want, name in ((cache.k, kc, "K"), (cache.v, vc, "V")):
        np.testing.assert_array_equal(got.view(torch.uint8).cpu().numpy(), want, err_msg=f"{what}: {name}")


def _run(hk, d, dtype, code, block, n_rows, steps, seed=0):
    """steps: (positions or None, row0, n, spread).  The cache begins empty and takes them one after the other."""
    sh = B.make_shape(hk, hk, d, B.BF16 if dtype is torch.bfloat16 else B.F32)
    cache = B.Cache8.empty(sh, n_rows, block, B.E4M3 if code == "e4m3" else B.INT8)
    nb = -(-n_rows // block)
    kc, vc = (np.zeros((n_rows, hk, d), np.uint8) for _ in range(2))
    ks, vs = (np.zeros((nb, hk), np.float32) for _ in range(2))
    for i, (pos, row0, n, spread) in enumerate(steps):
        what = f"step {i}: {hk} heads of {d}, {dtype}, {code}, blocks of {block}, {n} of {n_rows} rows"
        print(what, flush=True)
        k, v = _new(n, hk, d, dtype, seed + 10 * i, spread), _new(n, hk, d, dtype, seed + 10 * i + 1, spread * 3)
        reused, dev = torch.ones((n_rows,), dtype=torch.uint8).cuda(), torch.ones((hk, n_rows)).cuda()
        at = list(range(row0, row0 + n)) if pos is None else list(pos)
        sel = None if pos is None else torch.tensor(at, dtype=torch.int32).cuda()
        B.kvs_store_kv8(sh, cache, k.cuda(), v.cuda(), sel, row0, reused, dev)
        R.store(kc, ks, k.float().numpy(), at, block, code)
        R.store(vc, vs, v.float().numpy(), at, block, code)
        _same(cache, kc, ks, vc, vs, what)
        left = np.ones(n_rows, bool)
        left[[p for p in at if 0 <= p < n_rows]] = False
        np.testing.assert_array_equal(reused.cpu().numpy() != 0, left)
        np.testing.assert_array_equal(dev.cpu().numpy() != 0, np.broadcast_to(left, (hk, n_rows)))
    return cache


@pytest.mark.parametrize("code", ["e4m3", "int8"])
@pytest.mark.parametrize("block", [16, 32, 64, 128])
@pytest.mark.parametrize("hk,d,dtype", HEADS)
def test_a_prompt_then_recomputed_and_appended_rows(hk, d, dtype, block, code):
    rng = np.random.default_rng(block)
    n_rows = 300                                           # the last block ends inside
    picked = np.sort(rng.permutation(200)[:57])
    _run(hk, d, dtype, code, block, n_rows,
         [(None, 0, 200, 1.0),                             # a prompt
          (picked, 0, 57, 2.0),                            # some rows again: some scales grow
          ([200], 0, 1, 1.0), ([201], 0, 1, 8.0),          # a decode step's rows
          (None, 250, 50, 1.0),                            # up to the cache's end, from inside a block
          (None, 130, 1, 0.01),
          (list(range(40, 300)), 0, 260, 0.5)])            # a list of whole blocks: their scales are their own again


@pytest.mark.parametrize("code", ["e4m3", "int8"])
def test_lists(code):
    """Entries of a block in any order, equal ones, places outside the cache, requests in any order; one long list."""
    rng = np.random.default_rng(3)
    _run(2, 128, torch.bfloat16, code, 32, 1000,
         [([5, 3, 4, 31, 0], 0, 5, 1.0),
          ([7, 7, 7, 2, 7, 2], 0, 6, 1.0),                 # the last of equal entries counts
          ([-1, -5, 1000, 2000000000, 40, 41, -1], 0, 7, 1.0),
          ([900, 100, 500, 501, 320], 0, 5, 1.0),
          (sorted(int(x) for x in rng.integers(0, 32, 700)), 0, 700, 1.0),      # more entries than a block has rows
          (np.sort(rng.permutation(1000)[:400]), 0, 400, 1.0)])


@pytest.mark.parametrize("code", ["e4m3", "int8"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_odd_values(code, dtype):
    """Zeros, a block's scale at the least, huge values, a NaN or infinity: its block and head alone, for as long as a row is kept."""
    hk, d, block = 2, 64, 16
    sh = B.make_shape(hk, hk, d, B.BF16 if dtype is torch.bfloat16 else B.F32)
    x = torch.randn((64, hk, d), generator=torch.Generator().manual_seed(5)).to(dtype)
    x[0:16] = 0
    x[16:32, 0] *= 1e-38
    x[16:32, 1] *= 1e37
    x[33, 0, 5], x[50, 1, 7] = float("nan"), float("-inf")
    cache = B.Cache8.empty(sh, 64, block, B.E4M3 if code == "e4m3" else B.INT8)
    kc, ks = np.zeros((64, hk, d), np.uint8), np.zeros((4, hk), np.float32)
    B.kvs_store_kv8(sh, cache, x.cuda(), x.cuda(), None)
    R.store(kc, ks, x.float().numpy(), range(64), block, code)
    _same(cache, kc, ks, kc, ks, "first")
    assert np.isnan(ks[2, 0]) and np.isnan(ks[3, 1]) and not np.isnan(ks[2, 1]) and (ks[0] == 0).all()
    # a row of the block alone does not mend it, all of them do
    for rows in ([33], list(range(32, 48))):
        y = torch.ones((len(rows), hk, d), dtype=dtype)
        B.kvs_store_kv8(sh, cache, y.cuda(), y.cuda(), torch.tensor(rows, dtype=torch.int32).cuda())
        R.store(kc, ks, y.float().numpy(), rows, block, code)
        _same(cache, kc, ks, kc, ks, f"{len(rows)} rows")
        assert np.isnan(ks[2, 0]) == (len(rows) == 1)


def test_what_is_not_taken_stays():
    """Rows behind the last sequence and other blocks keep their bytes, whatever they are."""
    sh = B.make_shape(4, 2, 64, B.BF16)
    cache = B.Cache8.empty(sh, 100, 16)
    junk = torch.randint(0, 256, (2, 100, 2, 64), dtype=torch.uint8, generator=torch.Generator().manual_seed(1)).cuda()
    cache.k.view(torch.uint8).copy_(junk[0])
    cache.v.view(torch.uint8).copy_(junk[1])
    k = _new(20, 2, 64, torch.bfloat16, 1).cuda()
    B.kvs_store_kv8(sh, cache, k, k, None, 32)
    for got, was in ((cache.k, junk[0]), (cache.v, junk[1])):
        got = got.view(torch.uint8)
        assert torch.equal(got[:32], was[:32]) and torch.equal(got[64:], was[64:])
        # rows 52 .. 63 share a block whose scale was 0: they stand for zeros
        assert bool(((got[52:64] & 0x7F) == 0).all())
    assert bool((cache.k_scale[[0, 1, 4, 5, 6]] == 0).all()) and bool((cache.k_scale[2:4] > 0).all())


def test_replays_from_a_graph():
    sh = B.make_shape(8, 8, 128, B.BF16)
    caches = [B.Cache8.empty(sh, 512, 64) for _ in range(2)]
    k, pos = _new(100, 8, 128, torch.bfloat16, 2).cuda(), torch.arange(3, 503, 5, dtype=torch.int32).cuda()
    B.kvs_store_kv8(sh, caches[0], k, k, pos)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        B.kvs_store_kv8(sh, caches[1], k, k, pos)
    for i in range(3):
        g.replay()
        torch.cuda.synchronize()
        for x in ("k", "v", "k_scale", "v_scale"):
            a, b = (getattr(c, x).view(torch.uint8 if x in "kv" else torch.float32) for c in caches)
            assert torch.equal(a, b), (i, x)
        k.mul_(1.5)
        pos.add_(1)
        B.kvs_store_kv8(sh, caches[0], k, k, pos)
