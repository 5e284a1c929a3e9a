"""kvs_rotary: outputs that overlap an input or output are refused, whichever tensors they are; slices of one buffer that lie side by
side are not."""
import ctypes

import pytest
import torch

from paper_2503_16525_amd import binding as B

Q, K, QO, KO = 1 << 20, 1 << 21, 1 << 22, 1 << 23          # addresses; every call below fails its checks
WORD = {"q": b"overlaps q ", "k": b"overlaps k ", "out": b"overlaps k_out"}


@pytest.mark.parametrize("n,args,word", [
    # q rows are 1024 bytes, k rows 256; strides in elements of two bytes
    (10, dict(qo=K), "k"), (10, dict(ko=Q), "q"), (10, dict(ko=Q + 768, kos=512), "q"), (10, dict(ko=QO), "out"), (10, dict(ko=QO + 9 * 1024 + 768), "out"),
    (10, dict(qo=K - 9 * 1024 - 16), "k"), (10, dict(ko=Q + 9 * 1024), "q"), (1, dict(ko=Q + 768), "q"),
    (10, dict(qo=Q + 16), "q"), (10, dict(qo=Q - 1008), "q"), (10, dict(qs=2048, qos=2048, qo=Q + 1008), "q"), (10, dict(qs=2048, qos=2048, qo=Q + 4096 - 1008), "q"),
    (10, dict(qs=2048, qos=2048, qo=Q - 9 * 4096 + 16), "q"), (10, dict(qs=2048, qos=2048, qo=Q - 9 * 4096 - 1008), "q"),
    (10, dict(qs=2048, qos=4096, qo=Q + 2048), "q"),        # rows of another stride between
    (10, dict(q=Q, qs=2048, k=Q + 1024, ks=2048, qo=Q, qos=2048, ko=Q + 1024 - 16, kos=2048), "out"),
])
def test_refused(n, args, word):
    a = {**dict(q=Q, qs=512, k=K, ks=128, qo=QO, qos=512, ko=KO, kos=128), **args}
    lib, sh = B.load(), B.make_shape(4, 1, 128, B.BF16)
    rc = lib.kvs_rotary(ctypes.byref(sh), ctypes.byref(B.rotary_spec(128)), n, 1 << 16, None, a["q"], a["qs"], a["k"], a["ks"], a["qo"], a["qos"], a["ko"], a["kos"], None)
    assert rc == B.EINVAL and WORD[word] in lib.kvs_last_error() + b" ", lib.kvs_last_error()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("n", [1, 2, 300])
@pytest.mark.parametrize("rotary_dim", [128, 64, 36])
def test_slices_side_by_side(rotary_dim, n, dtype):
    """A buffer's columns hold Q, K and both outputs: in any order, in place, and outputs a row further down."""
    hq, hk, d = 4, 2, 128
    sh = B.make_shape(hq, hk, d, B.BF16 if dtype is torch.bfloat16 else B.F32)
    spec = B.rotary_spec(rotary_dim, base=500.0)
    pos = torch.arange(n, dtype=torch.int32).cuda() * 3
    x = torch.randn((n + 1, 2 * (hq + hk) * d), generator=torch.Generator().manual_seed(n)).to(dtype).cuda()

    def of(buf, at, heads, row=0):
        return buf[row:row + n, at * d:(at + heads) * d].view(n, heads, d)
    for q_at, k_at, qo_at, ko_at, down in ((0, 4, 6, 10, 0), (6, 4, 0, 10, 0), (2, 0, 8, 6, 1), (0, 4, 0, 10, 0), (0, 4, 0, 4, 0), (4, 0, 8, 2, 1)):
        q, k = of(x, q_at, hq), of(x, k_at, hk)
        want_q, want_k = torch.empty((n, hq, d), dtype=dtype, device="cuda"), torch.empty((n, hk, d), dtype=dtype, device="cuda")
        B.kvs_rotary(sh, spec, pos, None, q.contiguous(), k.contiguous(), want_q, want_k)
        buf = x.clone()
        B.kvs_rotary(sh, spec, pos, None, of(buf, q_at, hq), of(buf, k_at, hk), of(buf, qo_at, hq, down), of(buf, ko_at, hk, down))
        want = x.clone()
        of(want, qo_at, hq, down).copy_(want_q)
        of(want, ko_at, hk, down).copy_(want_k)
        assert torch.equal(buf, want), (q_at, k_at, qo_at, ko_at, down)
