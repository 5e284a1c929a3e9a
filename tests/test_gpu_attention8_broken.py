"""kvs_attention_kv8 over blocks whose scale is NaN: the rows that see one of their keys, and no others, become NaN, outputs and
log-sum-exps alike, whichever scale it is and whichever kernels the launch goes to."""
import pytest
import torch

import kv8_torch as T
from paper_2503_16525_amd import binding as B

pytestmark = pytest.mark.gpu


def _check(hq, hk, d, dtype, code, block, n, pos, seed, workspace):
    sh = B.make_shape(hq, hk, d, B.BF16 if dtype is torch.bfloat16 else B.F32)
    cache = T.normal_cache(n, hk, d, block, code, seed)
    q = (torch.randn((len(pos), hq, d), generator=torch.Generator().manual_seed(seed)) / d ** 0.5).to(dtype).cuda()
    at = torch.tensor(pos, dtype=torch.int32).cuda()
    ws = torch.empty((B.kvs_workspace_size("attention_kv8", sh, 1, n, len(pos)),), dtype=torch.uint8, device="cuda") if workspace else None
    grp, blk = hq // hk, (n // block) // 2
    for name in ("k_scale", "v_scale"):
        print(f"{hq}x{hk}x{d}, {dtype}, {code}/{block}, {len(pos)} of {n}, {name}, workspace {workspace}", flush=True)
        scale = getattr(cache, name)
        was = scale[blk, hk - 1].clone()
        scale[blk, hk - 1] = float("nan")
        out, lse = torch.full_like(q, 7.0), torch.full((len(pos), hq), 7.0, device="cuda")
        B.kvs_attention_kv8(sh, cache, [0], [n], [0, len(pos)], q, at, 1.0, out, lse, ws)
        scale[blk, hk - 1] = was
        broken = torch.zeros((len(pos), hq), dtype=torch.bool, device="cuda")
        broken[:, (hk - 1) * grp:] = (at >= blk * block)[:, None]
        assert bool(broken.any()) and not bool(broken.all())
        assert torch.equal(out.isnan(), broken[..., None].expand_as(out)), name
        assert torch.equal(lse.isnan(), broken), name
        assert bool(torch.isfinite(out[~broken]).all()) and bool(torch.isfinite(lse[~broken]).all())


@pytest.mark.parametrize("code,block", [("e4m3", 16), ("int8", 32), ("int8", 64)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("hq,hk,d", [(8, 2, 128), (4, 4, 64)])
def test_few_and_many_rows(hq, hk, d, dtype, code, block):
    _check(hq, hk, d, dtype, code, block, 500, [3, 499, 100, 300, 250], 1, True)
    _check(hq, hk, d, dtype, code, block, 500, list(range(2, 498, 3)), 2, False)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_key_ranges_in_pieces(dtype):
    _check(8, 2, 128, dtype, "e4m3", 32, 20000, [19999, 9000], 3, True)


@pytest.mark.parametrize("code", ["e4m3", "int8"])
def test_widened_contexts(code):
    _check(32, 8, 128, torch.bfloat16, code, 32, 6000, list(range(0, 6000, 2)), 4, True)
