"""kvs_store_paged: every byte of the pool, and the mass that it clears."""
import random

import pytest
import torch

import paged_ref as R
from paper_2503_16525_amd import binding as B

pytestmark = pytest.mark.gpu


def _bits(x):
    return x.view(torch.int16 if x.dtype is torch.bfloat16 else torch.int32)


def _check(hq, hk, d, dtype, page, reqs, seed, places=(0, 0), bad=(), listed=None, max_ctx=None, shared=None):
    c = R.Case(hq, hk, d, dtype, page, reqs, seed=seed, places=places)
    for b, p, x in bad:
        c.table[b, p] = x
    if shared:
        c.table[shared[0], shared[2]] = c.table[shared[1], shared[2]]
    cache, pages = c.on(max_ctx)
    cu, sel = c.of(listed)
    k_new, v_new = (torch.randn((c.n, hk, d), generator=c.gen).to(dtype).cuda() for _ in range(2))
    stride = pages.max_ctx + 3
    mass = torch.rand((len(c.lens), hk, stride), generator=c.gen).cuda()
    want_k, want_v, want_mass = c.k.clone(), c.v.clone(), mass.clone()
    for b, n in enumerate(c.lens):
        for t, p in enumerate(c.pos[b]):
            if not 0 <= p < min(n, pages.max_ctx):
                continue
            pid = int(c.table[b, p // page])
            if not 0 <= pid < c.n_pages:
                continue
            s = c.cu[b] + t
            want_k[pid, p % page], want_v[pid, p % page] = k_new[s], v_new[s]
            want_mass[b, :, p] = 0
    print(hq, hk, d, dtype, page, len(reqs), c.n, flush=True)
    B.kvs_store_paged(c.shape, cache, pages, cu, sel, k_new, v_new, mass)
    assert torch.equal(_bits(c.k), _bits(want_k)) and torch.equal(_bits(c.v), _bits(want_v))
    assert torch.equal(mass, want_mass)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("hk,d", [(1, 64), (2, 64), (4, 128), (8, 128), (3, 128), (64, 128), (17, 64)])
def test_tokens_of_all_kinds(hk, d, dtype):
    rng = random.Random(hk)
    _check(2 * hk, hk, d, dtype, 16, [(n, 1) for n in (0, 1, 15, 16, 17, 100)], seed=hk)
    _check(hk, hk, d, dtype, 32, [(70, 70)], seed=hk + 1)
    _check(hk, hk, d, dtype, 64, [(260, 33), (1, 1), (20, 0), (90, 90), (0, 3), (5, 9)], seed=hk + 2, places=(3, 5))
    _check(hk, hk, d, dtype, 16, [(200, sorted(rng.sample(range(200), 50))), (60, [5, 5, 5, 9, 59, 60, 1000, -1]), (33, [-3, 32])], seed=hk + 3, places=(0, 2))


def test_entries_that_name_no_page_and_contexts_cut_short():
    _check(4, 2, 64, torch.bfloat16, 16, [(200, 200), (90, [0, 20, 50, 89])], seed=1, bad=((0, 3, -1), (0, 11, 10 ** 6), (1, 1, -2 ** 31)))
    _check(4, 2, 64, torch.bfloat16, 16, [(200, list(range(190))), (90, [89])], seed=2, max_ctx=120)


def test_many_requests():
    rng = random.Random(5)
    lens = [rng.randrange(0, 70) for _ in range(300)]
    _check(4, 2, 64, torch.bfloat16, 16, [(n, 1) for n in lens], seed=3)
    _check(4, 2, 64, torch.bfloat16, 16, [(n, min(n, rng.choice([0, 0, 0, 1, 3, 40]))) for n in lens], seed=4, places=(1, 9))


def test_without_mass_and_from_a_graph():
    c = R.Case(8, 2, 128, torch.bfloat16, 16, [(40, 1), (17, 1)], seed=6, rest=0.0, width=8, spare=20)
    c.table[0, :8], c.table[1, :8] = torch.arange(8, dtype=torch.int32), torch.arange(8, 16, dtype=torch.int32)
    cache, pages = c.on(128)
    k_new, v_new = (torch.randn((2, 2, 128), device="cuda").bfloat16() for _ in range(2))
    call = lambda: B.kvs_store_paged(c.shape, cache, pages, None, None, k_new, v_new)
    call()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    want_k, want_v = c.k.clone(), c.v.clone()
    for step in range(5):
        c.ctx_len.add_(7)
        k_new.mul_(1.5)
        graph.replay()
        torch.cuda.synchronize()
        for b in range(2):
            p = int(c.ctx_len[b]) - 1
            want_k[int(c.table[b, p // 16]), p % 16], want_v[int(c.table[b, p // 16]), p % 16] = k_new[b], v_new[b]
        assert torch.equal(c.k, want_k) and torch.equal(c.v, want_v)


def test_rows_behind_32_bits():
    n_pages = 6 * 2 ** 30 // (16 * 2 * 128 * 2)
    k, v = (torch.zeros((n_pages, 16, 2, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    table = torch.tensor([[n_pages - 1, 0, n_pages - 2]], dtype=torch.int32, device="cuda")
    new = torch.randn((48, 2, 128), device="cuda").bfloat16()
    sh = B.make_shape(4, 2, 128, B.BF16)
    B.kvs_store_paged(sh, B.PagedCache(k, v), B.PageTable(table, torch.tensor([48], dtype=torch.int32, device="cuda"), 48), torch.tensor([0, 48], dtype=torch.int32, device="cuda"), None, new, -new)
    for i, p in enumerate((n_pages - 1, 0, n_pages - 2)):
        assert torch.equal(k[p], new[16 * i:16 * i + 16]) and torch.equal(v[p], -new[16 * i:16 * i + 16])
    assert not k[1:n_pages - 2].any() and not v[1:n_pages - 2].any()
