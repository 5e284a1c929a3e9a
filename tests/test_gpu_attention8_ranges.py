"""kvs_attention_kv8, launches that widen their contexts: the copy in the workspace holds the contexts' rows, wherever in the cache they
lie, so a workspace sized by them, or by the cache where contexts share rows, is enough."""
import pytest
import torch

import kv8_torch as T
from paper_2503_16525_amd import binding as B

pytestmark = pytest.mark.gpu

HQ, HK = 32, 8


def _case(code, block, n_rows, reqs, ws_rows, seed):
    """reqs: (first row, rows, positions)"""
    sh = B.make_shape(HQ, HK, 128, B.BF16)
    cache = T.normal_cache(n_rows, HK, 128, block, code, seed)
    off, ln = [r[0] for r in reqs], [r[1] for r in reqs]
    pos, cu = [], [0]
    for r in reqs:
        pos += [int(x) for x in r[2]]
        cu.append(len(pos))
    at = torch.tensor(pos, dtype=torch.int32).cuda()
    q = (torch.randn((len(pos), HQ, 128), generator=torch.Generator().manual_seed(seed)) / 128 ** 0.5).to(torch.bfloat16).cuda()
    size = B.kvs_workspace_size("attention_kv8", sh, len(ln), ws_rows, len(pos))
    ws = torch.full((size + 4096,), 255, dtype=torch.uint8, device="cuda")
    out, lse = torch.full_like(q, 7.0), torch.full((len(pos), HQ), 7.0, device="cuda")
    print(f"{code}/{block}, {len(ln)} contexts, {len(pos)} tokens, a workspace for {ws_rows} of {n_rows} rows: {size} bytes", flush=True)
    B.kvs_attention_kv8(sh, cache, off, ln, cu, q, at, 1.0, out, lse, ws[:size])
    assert bool((ws[size:] == 255).all())
    assert bool((ws[size - 8192:size] != 255).any()), "the contexts were not widened"
    want, want_lse, mag, dots, _ = T.attention(q, at, cache, off, ln, cu, 1.0)
    # a weight and the output rounded to bf16, 2^-8 each: sum |w| |v - out| <= 2 mag; scores in fp32 as elsewhere
    fp32 = (132 * dots + 64 + max(ln)) * 2.0 ** -24
    tol = 2.0 ** -8 * (2 * mag + want.abs()) + 2 * fp32 * mag + 1e-30
    assert bool(((out.double() - want).abs() <= tol).all())
    empty = torch.isneginf(want_lse)
    assert torch.equal(torch.isneginf(lse), empty)
    assert bool(((lse.double() - want_lse)[~empty].abs() <= fp32 + 2.0 ** -22 * want_lse[~empty].abs()).all())


@pytest.mark.parametrize("code,block", [("e4m3", 32), ("int8", 128)])
def test_contexts_far_apart(code, block):
    reqs = [(96000 - 5200, 5200, range(0, 5200, 2)), (16, 5207, range(1, 5207, 2)), (48000, 40, [39, -1, 0])]
    _case(code, block, 96000, reqs, sum(r[1] for r in reqs), 1)


@pytest.mark.parametrize("code,block", [("e4m3", 16), ("int8", 64)])
def test_contexts_that_share_rows(code, block):
    """The same prompt under several requests, contexts inside others and next to others, in any order; together more rows than the cache has."""
    reqs = [(0, 6000, range(0, 6000, 3)), (3200, 2800, range(0, 2800, 2)), (0, 6000, range(1, 6000, 3)), (1600, 1601, range(0, 1601, 2)),
            (6000, 17, [16, 3]), (6032, 1, [0]), (6048, 31, [-5, 30, 100]), (3216, 16, [15])]
    _case(code, block, 6080, reqs, 6080, 2)


def test_a_longer_list_than_one_launch_describes():
    """66 requests: the second launch's begin behind the first's rows."""
    reqs = [(2000 * (b % 40), 1999 - 16 * (b % 7), range(b % 5, 1800, 3)) for b in range(64)] + [(0, 80000, range(7, 80000, 61)), (64000, 15990, range(3, 15990, 5))]
    _case("e4m3", 32, 80000, reqs, 64 * 1999 + 96000, 3)
