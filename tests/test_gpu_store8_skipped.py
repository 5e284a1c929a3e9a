"""kvs_store_kv8, lists with entries that are skipped: they may stand between the entries of one block, one or thousands of them, and change
nothing.  Bit for bit against the definition."""
import numpy as np
import pytest
import torch

import kv8_ref as R
from paper_2503_16525_amd import binding as B
from test_gpu_store8 import _new, _run, _same

pytestmark = pytest.mark.gpu


def _with_gaps(rng, at, gaps, n_rows):
    """`at` with gaps[i] skipped entries before its entry i, and gaps[-1] behind the last"""
    out = []
    for p, g in zip(list(at) + [None], gaps):
        out += [int(x) for x in rng.choice([-1, -7, n_rows, 2 ** 31 - 1], g)]
        if p is not None:
            out.append(int(p))
    return out


@pytest.mark.parametrize("code", ["e4m3", "int8"])
@pytest.mark.parametrize("hk,d,dtype", [(8, 128, torch.bfloat16), (1, 64, torch.float32), (20, 128, torch.float32)])
@pytest.mark.parametrize("block", [16, 128])
def test_gaps_inside_blocks(hk, d, dtype, block, code):
    rng = np.random.default_rng(block + hk)
    n_rows = 700
    steps = []
    for k, most in ((300, 3), (40, 80), (12, 700), (5, 3000), (1, 70)):
        at = np.sort(rng.permutation(n_rows)[:k])
        gaps = rng.integers(0, most + 1, k + 1) * (rng.random(k + 1) < 0.7)
        full = _with_gaps(rng, at, gaps, n_rows)
        steps.append((full, 0, len(full), 1.0 + len(steps)))
    # whole blocks, a gap behind every entry; the same entry again behind a gap counts as the last of equals
    full = _with_gaps(rng, range(3 * block), [1] * (3 * block) + [0], n_rows)
    steps.append((full, 0, len(full), 0.3))
    again = [5, -1, 6, -1, 5] + [-1] * 1500 + [6, n_rows, 5]
    steps.append((again, 0, len(again), 2.0))
    _run(hk, d, dtype, code, block, n_rows, steps, seed=7)


@pytest.mark.parametrize("lead", [0, 1, 63, 64, 65, 1023, 1024, 1025, 1087, 1088, 1089, 5000])
def test_gaps_of_every_reach(lead):
    """A run that is followed, and looked back for, over gaps that end at and beside what a wave asks for at once."""
    for block, hk in ((32, 2), (128, 8)):
        at = [40] + [-1] * lead + [41, 40 + block] + [-1] * lead + [41 + block] + [-1] * lead
        _run(hk, 64, torch.bfloat16, "int8", block, 400, [(list(range(400)), 0, 400, 0.1), (at, 0, len(at), 3.0)], seed=lead)


def test_padded_batch_of_requests_that_share_blocks():
    """Decode steps of a padded batch in ascending order: ended requests between live ones of the same block."""
    rng = np.random.default_rng(2)
    for step in range(3):
        at = [(-1 if rng.random() < 0.6 else 6 * b + step) for b in range(160)]
        _run(8, 128, torch.bfloat16, "e4m3", 64, 1000, [(None, 0, 1000, 0.5), (at, 0, len(at), 2.0 + step)], seed=step)


def test_nothing_is_stored_for_a_list_of_skipped_entries():
    sh = B.make_shape(2, 2, 64, B.BF16)
    cache = B.Cache8.empty(sh, 100, 32)
    k = _new(3000, 2, 64, torch.bfloat16, 1).cuda()
    B.kvs_store_kv8(sh, cache, k, k, torch.full((3000,), -1, dtype=torch.int32).cuda())
    zeros, ones = np.zeros((100, 2, 64), np.uint8), np.zeros((4, 2), np.float32)
    _same(cache, zeros, ones, zeros, ones, "skipped")
