"""Contexts that have outgrown what the host promised (max_ctx, or the table's width): new tokens at a context's end stand where the
length says, behind the rows that are taken.  They overwrite none of those, and see what the last one sees."""
import pytest
import torch

import paged_many as M
import paged_ref as R
from paper_2503_16525_amd import binding as B
from test_gpu_paged_attention import _attend, _parts
from test_gpu_paged_mass import _check as check_mass

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


def _grown(hq, hk, d, dtype, page, reqs, taken, seed=0):
    """A case whose requests have grown to reqs' lengths, of which `taken` rows are taken"""
    c = R.Case(hq, hk, d, dtype, page, reqs, seed=seed)
    c.lens = [min(n, taken) for n in c.lens]
    c.slots = [s[:taken] for s in c.slots]
    return c


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("listed", [False, True])
def test_a_store_overwrites_nothing(dtype, listed):
    """A decode step behind the promise stores nothing; a chunk's tokens that are inside are stored where they belong."""
    for reqs, taken in (([(200, 1), (90, 1), (121, 1)], 120), ([(200, 100), (90, 20), (150, 10), (120, 120)], 120)):
        c = R.Case(4, 2, 64, dtype, 16, reqs, seed=3)
        k_new, v_new = (torch.randn((c.n, 2, 64), generator=c.gen).to(dtype).cuda() for _ in range(2))
        mass = torch.rand((len(reqs), 2, taken), generator=c.gen).cuda()
        want_k, want_v, want_mass = c.k.clone(), c.v.clone(), mass.clone()
        for b, p in enumerate(c.pos):
            for t, i in enumerate(p):
                if i < taken:
                    to = (int(c.table[b, i // 16]), i % 16)
                    want_k[to], want_v[to], want_mass[b, :, i] = k_new[c.cu[b] + t], v_new[c.cu[b] + t], 0.0
        cache, pages = c.on(taken)
        cu, sel = c.of(listed)
        B.kvs_store_paged(c.shape, cache, pages, cu, sel, k_new, v_new, mass)
        bits = torch.int16 if dtype is BF16 else torch.int32
        assert torch.equal(c.k.view(bits), want_k.view(bits)) and torch.equal(c.v.view(bits), want_v.view(bits)) and torch.equal(mass, want_mass)


def test_a_store_behind_the_tables_width():
    c = R.Case(4, 2, 64, BF16, 16, [(32, 1)], seed=4, rest=0.5)
    c.ctx_len.fill_(2 ** 31 - 1)
    before = c.k.clone(), c.v.clone()
    cache, pages = c.on(10 ** 6)
    new = torch.ones((1, 2, 64), dtype=BF16, device="cuda")
    B.kvs_store_paged(c.shape, cache, pages, None, None, new, new)
    assert torch.equal(c.k, before[0]) and torch.equal(c.v, before[1])


@pytest.mark.parametrize("window,n_first", [(0, 0), (40, 5), (300, 0)])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_attention(dtype, window, n_first):
    for reqs, taken in (([(200, 1), (90, 1), (121, 1)], 120), ([(200, 100), (90, 20), (150, 10), (120, 120), (500, 3)], 120), ([(3000, 400)], 2800)):
        c = _grown(8, 2, 128, dtype, 16, reqs, taken, seed=taken)
        ref = R.attention(c, window, n_first)
        for listed in (False, True):
            for ws_bytes in (None, 0):
                out, lse = _attend(c, window, n_first, max_ctx=taken, listed=listed, ws_bytes=ws_bytes)
                R.check_attention(c, out, lse, ref, _parts(c), f"{reqs}, {taken} taken, listed {listed}")


@pytest.mark.parametrize("window,n_first", [(0, 0), (400, 5)])
def test_attention_of_many_rows(window, n_first):
    for reqs, taken in (([(3000, 400)], 2800), ([(900, 300), (700, 700), (200, 50)], 650)):
        c = _grown(8, 2, 128, BF16, 16, reqs, taken, seed=taken)
        ref = R.attention(c, window, n_first)
        with M.forced(1) as lib:
            assert M.choice(lib, c.shape, 16, len(reqs), taken, c.n, window=window, n_first=n_first)[0]
            out, lse = _attend(c, window, n_first, max_ctx=taken)
        R.check_attention(c, out, lse, ref, 1, f"{reqs}, {taken} taken")


@pytest.mark.parametrize("window,n_first", [(0, 0), (40, 5)])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_mass(dtype, window, n_first):
    for reqs, taken in (([(200, 1), (90, 1), (121, 1)], 120), ([(400, 300), (90, 90), (250, 100), (220, 220)], 220)):
        check_mass(_grown(8, 2, 128, dtype, 16, reqs, taken, seed=taken), "grown", window, n_first, max_ctx=taken)
