"""kvs_rotary with very many heads: up to 4095 of them turn, more are refused."""
import ctypes

import pytest
import torch

from paper_2503_16525_amd import binding as B


@pytest.mark.parametrize("hq,hk", [(4095, 1), (4096, 4096), (1 << 29, 1 << 29), (1 << 30, 1), (2147483647, 1)])
@pytest.mark.parametrize("rotary_dim", [128, 8])
def test_refused(hq, hk, rotary_dim):
    lib, sh, at = B.load(), B.make_shape(hq, hk, 128, B.BF16), 1 << 40
    rc = lib.kvs_rotary(ctypes.byref(sh), ctypes.byref(B.rotary_spec(rotary_dim)), 1, 1 << 16, None, at, hq * 128, None, 0, at, hq * 128, None, 0, None)
    assert rc == B.EUNSUPPORTED and b"heads" in lib.kvs_last_error()


@pytest.mark.gpu
@pytest.mark.parametrize("hq,hk", [(4094, 1), (2047, 2047), (3000, 1000)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rotary_dim", [128, 64, 34])
def test_the_most(hq, hk, rotary_dim, dtype):
    """Every head turns as the others do."""
    n, d = 3, 128
    sh, few = (B.make_shape(h, k, d, B.BF16 if dtype is torch.bfloat16 else B.F32) for h, k in ((hq, hk), (1, 1)))
    spec, pos = B.rotary_spec(rotary_dim), torch.tensor([5, 0, 70000], dtype=torch.int32).cuda()
    x = torch.randn((n, 1, d), generator=torch.Generator().manual_seed(hq)).to(dtype).cuda()
    want = torch.empty_like(x)
    B.kvs_rotary(few, spec, pos, None, x, None, want, None)
    q, k = x.expand(n, hq, d).contiguous(), x.expand(n, hk, d).contiguous()
    q_out, k_out = torch.empty_like(q), torch.empty_like(k)
    B.kvs_rotary(sh, spec, pos, None, q, k, q_out, k_out)
    assert torch.equal(q_out, want.expand_as(q)) and torch.equal(k_out, want.expand_as(k))
