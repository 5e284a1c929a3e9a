"""kvs_deviation_kv8 against the same sums in 64 bits on what the cache stands for."""
import numpy as np
import pytest
import torch

import kv8_ref as R
from paper_2503_16525_amd import binding as B

pytestmark = pytest.mark.gpu


def _check(hk, d, dtype, code, block, row0, n, mode, weighted, mask, seed):
    n_rows = row0 + n + 7
    cache = R.make(n_rows, hk, d, block, code, seed)
    gpu = R.on_gpu(B, cache, block, code)
    kh, vh = R.held(cache[0], cache[1], block, code)[row0:row0 + n], R.held(cache[2], cache[3], block, code)[row0:row0 + n]
    rng = np.random.default_rng(seed + 1)
    noise = np.exp(rng.normal(-3, 1.5, (n, 1, 1)))
    kf, vf = (torch.from_numpy((x + noise * rng.normal(size=x.shape)).astype(np.float32)).to(dtype) for x in (kh, vh))
    alpha = rng.uniform(0.1, 3, (hk, n)).astype(np.float32) if weighted else None
    reused = (rng.random(n) < 0.7).astype(np.uint8) if mask else None
    sh = B.make_shape(2 * hk, hk, d, B.BF16 if dtype is torch.bfloat16 else B.F32)
    up = lambda x: None if x is None else torch.from_numpy(x).cuda()
    dk, dv, score = torch.full((hk, n), 7.0).cuda(), torch.full((hk, n), 7.0).cuda(), torch.full((n,), 7.0).cuda()
    B.kvs_deviation_kv8(sh, gpu, row0, n, kf.cuda() if mode else None, vf.cuda(), up(reused), up(alpha), mode, dk if mode else None, dv, score)
    want_k, want_v = np.abs(kf.double().numpy() - kh).sum(-1).T, np.abs(vf.double().numpy() - vh).sum(-1).T
    want = want_v + want_k if mode else want_v
    want = (want * alpha.astype(np.float64) if weighted else want).sum(0)
    # a term is rounded once, and passes through at most 12 sums of positive numbers; a score through hk + 2 more
    rel = 14 * 2.0 ** -24
    np.testing.assert_allclose(dv.cpu().numpy(), want_v, rtol=rel)
    if mode:
        np.testing.assert_allclose(dk.cpu().numpy(), want_k, rtol=rel)
    got = score.cpu().numpy()
    left = np.ones(n, bool) if reused is None else reused != 0
    assert np.isneginf(got[~left]).all()
    np.testing.assert_allclose(got[left], want[left], rtol=rel + (hk + 2) * 2.0 ** -24)


@pytest.mark.parametrize("code", ["e4m3", "int8"])
@pytest.mark.parametrize("hk,d,dtype", [(8, 128, torch.bfloat16), (4, 64, torch.float32), (3, 128, torch.float32), (1, 64, torch.bfloat16), (64, 64, torch.bfloat16)])
@pytest.mark.parametrize("block,row0,n", [(16, 0, 1), (32, 5, 333), (64, 17, 31), (128, 64, 8200)])
def test_scores(hk, d, dtype, code, block, row0, n):
    if n * hk > 70000:
        n = 8200 // 16
    _check(hk, d, dtype, code, block, row0, n, B.SCORE_V, False, True, n + hk)
    _check(hk, d, dtype, code, block, row0, n, B.SCORE_KV, True, False, n + hk + 1)


def test_blocks_that_hold_nothing_and_broken_ones():
    """A scale of 0 stands for zeros whatever the codes; a NaN scale reaches its block's tokens and no others."""
    sh = B.make_shape(2, 2, 128, B.BF16)
    cache = B.Cache8.empty(sh, 64, 16)
    cache.v.view(torch.uint8).fill_(0xFF)                  # e4m3's NaN
    vf = torch.ones((64, 2, 128), dtype=torch.bfloat16).cuda()
    dv, score = torch.empty((2, 64)).cuda(), torch.empty((64,)).cuda()
    cache.v_scale[2, 1] = float("nan")
    B.kvs_deviation_kv8(sh, cache, 0, 64, None, vf, None, None, B.SCORE_V, None, dv, score)
    want = np.full((2, 64), 128.0)
    want[1, 32:48] = np.nan
    np.testing.assert_array_equal(dv.cpu().numpy(), want)
    np.testing.assert_array_equal(np.isnan(score.cpu().numpy()), np.isnan(want[1]))
