"""Partial attention in launches whose softmax reference moves or that are cut into pieces: what a row has collected before a reference
moves, or in another piece, keeps its weight.  Scores are whole powers of two (in base 2), which bf16 holds, against 64 bits."""
import math

import pytest
import torch

from paper_2503_16525_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda"


def _run(hq, hk, n, pos, level, v, seed, workspace=True):
    """Every query head scores `level` (base 2) at every key.  -> out, lse, reference of both in 64 bits (KV heads' rows)"""
    d, k = 128, pos.numel()
    kk = torch.zeros((n, hk, d), device=DEV)
    kk[:, :, 0], kk[:, :, 1] = (level / 64).floor()[:, None], (level % 64)[:, None]
    q = torch.zeros((k, hq, d), device=DEV)
    q[:, :, 0], q[:, :, 1] = 64, 1
    kk, q, v = kk.to(torch.bfloat16), q.to(torch.bfloat16), v.to(torch.bfloat16)
    sh = B.make_shape(hq, hk, d, B.BF16)
    ws = torch.empty(B.kvs_workspace_size("partial_attention", sh, 1, n, k), dtype=torch.uint8, device=DEV) if workspace else None
    out, lse = torch.full((k, hq, d), 7.0, dtype=torch.bfloat16, device=DEV), torch.full((k, hq), 7.0, device=DEV)
    B.kvs_partial_attention(sh, [0], [n], [0, k], q, pos, kk, v, math.log(2), out, lse, ws)
    some = torch.tensor(sorted({0, 1, k // 3, k // 2, k - 2, k - 1}), device=DEV)
    s = torch.where(torch.arange(n, device=DEV)[None] <= pos[some, None], level.double()[None] * math.log(2), -torch.inf)
    w, z = torch.softmax(s, 1), torch.logsumexp(s, 1)
    for g in range(hk):
        ref = (w @ v[:, g].double())[:, None]
        mag = (w @ v[:, g].double().abs())[:, None]
        got = out[some, g * (hq // hk):(g + 1) * (hq // hk)].double()
        # a weight's rounding in numerator and normaliser, 2^-8 each, the scale's in fp32 (2^-24 of a score of up to 200, twice), the output's half step
        tol = 2.0 ** -8 * ref.abs() + mag * (2 * 2.0 ** -8 + 2 * 2.0 ** -16)
        used = float(((got - ref).abs() / tol).max())
        assert used <= 1, f"KV head {g}: {used} of the tolerance"
    # (log2 e and ln 2 in fp32, each off by 2^-24 of a result of up to 140, and the result's own)
    off, tol = float((lse[some].double() - z[:, None]).abs().max()), 2.0 ** -24 * 4 * float(z.abs().max() + 1) + 1e-5
    assert off <= tol, f"log-sum-exp off by {off}, {tol} allowed"


@pytest.mark.parametrize("rise", [9, 11, 12, 13, 14, 16, 20, 40, 70])
def test_a_reference_that_moves_keeps_what_came_before(rise):
    """A thousand keys stand so far above the first tile that their sum is just below what moves the reference; one key that comes after them does
    that.  Up to 24 % of a row's weight is what came before."""
    print(f"rise of {rise}", flush=True)
    n, k = 49200, 1600                                       # K and V beyond the last-level cache
    gen = torch.Generator(device=DEV).manual_seed(rise)
    level = torch.zeros((n,), device=DEV)
    level[32:1032] = 115
    level[1100] = 115 + rise
    v = torch.randn((n, 8, 128), generator=gen, device=DEV).abs() + 1
    v[1100] = -v[1100]
    _run(64, 8, n, torch.arange(n - k * 30, n, 30, device=DEV, dtype=torch.int32), level, v, rise)


@pytest.mark.parametrize("hq,hk,n,k", [(32, 8, 8192, 738), (28, 4, 12000, 481), (32, 8, 3000, 200)])
@pytest.mark.parametrize("first,others", [(150, 130), (150, 125), (99, 60), (140, 128), (60, 190), (105, 20)])
def test_pieces_whose_first_tiles_lie_far_apart(hq, hk, n, k, first, others):
    """Launches that are cut into pieces: the first piece's logits begin at 0 and rise to `first` in one key, those of the context's second half
    are all `others`.  Each piece counts by what it holds, wherever its reference stands."""
    print(f"{k} of {n} on {hq}:{hk}, {first} beside {others}", flush=True)
    gen = torch.Generator(device=DEV).manual_seed(first)
    level = torch.zeros((n,), device=DEV)
    level[100], level[n // 2:] = first, others
    v = torch.randn((n, hk, 128), generator=gen, device=DEV).abs() + 1
    v[100] = -v[100]
    pos = (torch.arange(k, device=DEV) * n // k).int()
    _run(hq, hk, n, pos, level, v, first)
    _run(hq, hk, n, pos, level, v, first, workspace=False)
