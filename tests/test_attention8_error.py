"""kvs_attention_kv8: how far outputs are from 64 bits in norm, which the worst-case bounds of the other tests leave open.  A model of the
arithmetic on the CPU shows that these bounds tell one bf16 number more or fewer apart; the kernels then have to keep them.

fp32.  A score is a chain of 3 d / 16 <= 24 products added in fp32, so its error is about sqrt(24) 2^-25 of partial sums of 1 to 3: 2 to 7 times
2^-24; a weight's own, its product and the sums add a few more: 2^-20 is 16 times 2^-24.  Two bf16 numbers in place of three hold a
number to 2^-17 at worst, 2^-18.3 in root mean square, which a sum of independent errors carries into the result: 50 times 2^-24.
bf16.  Rounding the result once leaves an error r.  Weights held to 2^-17 add nothing that shows (up to 1.1 r allowed).  Weights rounded to
bf16 add an error of r in every weight: sqrt(r^2 + r^2) = 1.41 r together where many keys count, 1.29 r where three do.  A V rounded too would
be sqrt(3) r = 1.73; 1.57 lies between."""
import pytest
import torch

import kv8_torch as T
from paper_2503_16525_amd import binding as B

FP32, TWO, ONE = 2.0 ** -20, 1.1, 1.57


def _ratio(out, want):
    return T.off_by(out, want) / T.off_by(want.to(torch.bfloat16), want)


def _split(x, parts):
    """bf16 numbers (as fp32) that add up to x to 8 bits each"""
    out = []
    for _ in range(parts):
        out.append(x.to(torch.bfloat16).float())
        x = x - out[-1]
    return out


def _codes(n, d, block, seed, large=()):
    gen = torch.Generator().manual_seed(seed)
    x = torch.randn((2, n, d), generator=gen)
    toward = torch.randn((d,), generator=gen) / d ** 0.5
    for i in large:                                        # keys of nearly the same large score for a query along `toward`
        x[0, i] = 12 * toward + 0.3 * x[0, i]
    scale = (x.abs().amax(-1).view(2, -1, block).amax(-1) / 127).repeat_interleave(block, 1)
    return (x / scale[..., None]).round(), scale, toward


def _model(q, codes, scale, nq, np_, dtype):
    """one KV head's rows with Q in nq bf16 numbers and weights in np_"""
    s = sum(part @ codes[0].T for part in _split(q, nq)) * scale[0] if nq > 1 else (q @ codes[0].T) * scale[0]
    p = torch.exp(s - s.amax(1, keepdim=True))
    y = _split(p * scale[1], np_)
    total = p.sum(1) if np_ > 1 else (y[0] / scale[1]).sum(1)
    return (sum(part @ codes[1] for part in y) / total[:, None]).to(dtype)


@pytest.mark.parametrize("n,large", [(128, ()), (3008, ()), (512, (100, 200, 300))])
def test_the_bounds_tell_the_arithmetic_apart(n, large):
    d = 128
    codes, scale, toward = _codes(n, d, 32, n, large)
    gen = torch.Generator().manual_seed(1)
    q = torch.randn((64, d), generator=gen) / d ** 0.5
    if large:
        q = q + toward                                     # these keys take nearly all weight
    held = (codes * scale[..., None]).double()

    def want(x):
        return torch.softmax(x.double() @ held[0].T, 1) @ held[1]
    if not large:                                          # (scores of 1 to 3: the error grows with them)
        assert T.off_by(_model(q, codes, scale, 3, 3, torch.float32), want(q)) <= FP32
        assert T.off_by(_model(q, codes, scale, 2, 3, torch.float32), want(q)) > FP32
        assert T.off_by(_model(q, codes, scale, 3, 2, torch.float32), want(q)) > FP32
    q = q.to(torch.bfloat16).float()
    assert _ratio(_model(q, codes, scale, 1, 2, torch.bfloat16), want(q)) <= TWO
    assert TWO < _ratio(_model(q, codes, scale, 1, 1, torch.bfloat16), want(q)) <= ONE
    if not large:                                          # V rounded too
        p = torch.exp((q @ codes[0].T) * scale[0]).to(torch.bfloat16).float()
        out = (p @ held[1].to(torch.bfloat16).float()) / p.sum(1)[:, None]
        assert _ratio(out.to(torch.bfloat16), want(q)) > ONE


def _run(hq, hk, d, dtype, code, block, n, rows, seed, workspace, spread=1.0):
    sh = B.make_shape(hq, hk, d, B.BF16 if dtype is torch.bfloat16 else B.F32)
    cache = T.normal_cache(n, hk, d, block, code, seed)
    gen = torch.Generator().manual_seed(seed)
    q = (torch.randn((rows, hq, d), generator=gen) * spread / d ** 0.5).to(dtype).cuda()
    pos = torch.sort(torch.randint(n // 2, n, (rows,), generator=gen)).values.to(torch.int32).cuda()
    ws = torch.empty((B.kvs_workspace_size("attention_kv8", sh, 1, n, rows),), dtype=torch.uint8, device="cuda") if workspace else None
    out, lse = torch.full_like(q, 7.0), torch.full((rows, hq), 7.0, device="cuda")
    B.kvs_attention_kv8(sh, cache, [0], [n], [0, rows], q, pos, 1.0, out, lse, ws)
    want = T.attention(q, pos, cache, [0], [n], [0, rows], 1.0)[0]
    what = f"{hq}x{hk}x{d} {dtype} {code}/{block} {rows} of {n}, workspace {workspace}"
    print(what, T.off_by(out, want), _ratio(out, want), flush=True)
    return T.off_by(out, want), _ratio(out, want)


@pytest.mark.gpu
@pytest.mark.parametrize("code", ["e4m3", "int8"])
@pytest.mark.parametrize("hq,hk,d", [(8, 2, 128), (4, 4, 64)])
@pytest.mark.parametrize("n,rows,workspace", [(33, 5, False), (500, 77, False), (3001, 200, True), (20000, 3, True)])
def test_fp32(n, rows, workspace, hq, hk, d, code):
    assert _run(hq, hk, d, torch.float32, code, 32, n, rows, n, workspace)[0] <= FP32


@pytest.mark.gpu
@pytest.mark.parametrize("code", ["e4m3", "int8"])
@pytest.mark.parametrize("hq,hk,d", [(32, 4, 128), (8, 8, 64)])
@pytest.mark.parametrize("n,rows,workspace", [(33, 4, False), (500, 4, False), (3001, 2, True), (30000, 1, True)])
@pytest.mark.parametrize("spread", [1.0, 3.0])
def test_bf16_single_tokens(spread, n, rows, workspace, hq, hk, d, code):
    """One row block a request: two bf16 numbers a weight, also where a few keys have most of it."""
    assert _run(hq, hk, d, torch.bfloat16, code, 32, n, rows, n, workspace, spread)[1] <= TWO


@pytest.mark.gpu
@pytest.mark.parametrize("code", ["e4m3", "int8"])
@pytest.mark.parametrize("hq,hk,n,rows,workspace", [(32, 8, 3001, 200, False), (32, 8, 9000, 150, True), (32, 8, 9000, 3000, True), (28, 4, 12000, 2500, True)])
def test_bf16_many_rows(hq, hk, n, rows, workspace, code):
    """Several row blocks, and contexts that are widened first (the last two): one bf16 number a weight, V as it is held."""
    assert _run(hq, hk, 128, torch.bfloat16, code, 32, n, rows, n, workspace)[1] <= ONE
