"""A cache in 8 bits that is filled a row at a time, as decode steps do: its scale grows with the rows, and what is held is rounded again
each time.  How far it may then be from the rows (the definition, on the CPU), and that the kernel does just that."""
import numpy as np
import pytest
import torch

import kv8_ref as R
from paper_2503_16525_amd import binding as B


def _rows(n, hk, d, rising, block, seed):
    rng = np.random.default_rng(seed)
    x = rng.normal(0, 1, (n, hk, d)).astype(np.float32)
    return x * (1 + np.arange(n) % block / 8).astype(np.float32)[:, None, None] if rising else x


@pytest.mark.parametrize("code", ["e4m3", "int8"])
@pytest.mark.parametrize("block", [16, 128])
@pytest.mark.parametrize("rising", [False, True])
def test_error_of_appended_rows(rising, block, code):
    """Stored once, and rounded again with every growth behind that: each time by half a step at most, of the scale of that time, which is no larger
    than the last.  A step of int8 is the scale; of e4m3 at most 2^-3 of the value, which is at most 1 + 2^-4 times as large as it was for each
    rounding, and 2^-9 scales below 2^-6 of them.  2^-20 for the fp32 arithmetic of a rounding."""
    n, hk, d = 2 * block, 2, 64
    x = _rows(n, hk, d, rising, block, 1)
    codes, scale = np.zeros((n, hk, d), np.uint8), np.zeros((2, hk), np.float32)
    roundings = np.zeros((n, hk), np.int64)
    for i in range(n):
        old = scale.copy()
        R.store(codes, scale, x[i:i + 1], [i], block, code)
        blk = i // block
        roundings[blk * block:i, scale[blk] != old[blk]] += 1
        roundings[i] += 1
    off = np.abs(R.held(codes, scale, block, code) - x)
    s = scale.astype(np.float64).repeat(block, 0)[:, :, None]
    k = roundings[:, :, None]
    step = s if code == "int8" else np.maximum(np.abs(x) * 2.0 ** -3 * (1 + 2.0 ** -4) ** k, s * 2.0 ** -9)
    assert (off <= k * (step / 2 + 2.0 ** -20 * np.abs(x).max())).all()
    once, scale = np.zeros_like(codes), np.zeros_like(scale)
    R.store(once, scale, x, range(n), block, code)
    at_once = np.linalg.norm(R.held(once, scale, block, code) - x)
    # in norm: errors of independent roundings, the earlier ones in smaller steps
    assert np.linalg.norm(off) <= at_once * np.sqrt(roundings.max())


@pytest.mark.gpu
@pytest.mark.parametrize("code", ["e4m3", "int8"])
@pytest.mark.parametrize("block", [16, 128])
def test_decode_steps_of_many_requests(block, code):
    """A row each for 70 requests a step, each in blocks of its own, some of them ended: every byte as the definition has it."""
    n_req, hk, d = 70, 2, 64
    n = n_req * block
    sh = B.make_shape(hk, hk, d, B.F32)
    cache = B.Cache8.empty(sh, n, block, B.E4M3 if code == "e4m3" else B.INT8)
    x = _rows(n, hk, d, True, block, 2)
    codes, scale = np.zeros((n, hk, d), np.uint8), np.zeros((n_req, hk), np.float32)
    print(f"{code}/{block}", flush=True)
    for step in range(0, block, 1 if block == 16 else 9):
        at = [b * block + step if (b * 7 + step) % 5 else -1 for b in range(n_req)]
        new = np.stack([x[p] if p >= 0 else np.full((hk, d), 1e9, np.float32) for p in at])
        k = torch.from_numpy(new).cuda()
        B.kvs_store_kv8(sh, cache, k, k, torch.tensor(at, dtype=torch.int32).cuda())
        R.store(codes, scale, new, at, block, code)
    for got, want in ((cache.k, codes), (cache.v, codes)):
        np.testing.assert_array_equal(got.view(torch.uint8).cpu().numpy(), want)
    for got in (cache.k_scale, cache.v_scale):
        np.testing.assert_array_equal(got.cpu().numpy(), scale)
