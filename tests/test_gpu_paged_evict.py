"""kvs_evict_paged: which rows stay, and every byte of what is copied."""
import random

import pytest
import torch

import paged_ref as R
from paper_2503_16525_amd import binding as B

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


def _bits(x):
    return x.view(torch.int16 if x.dtype is BF16 else torch.int32)


def _check(hq, hk, d, dtype, page, lens, keep, n_first, n_recent, seed, weigh=None, max_ctx=None, max_keep=None, bad_new=(), bad_old=(), same_len=False):
    c = R.Case(hq, hk, d, dtype, page, [(n, 0) for n in lens], seed=seed, spare=sum(-(-max(k, 0) // page) + 1 for k in keep) + 3)
    cache, pages = c.on(max_ctx)
    lens = [min(n, pages.max_ctx) for n in lens]
    max_keep = max(max(keep), 1) if max_keep is None else max_keep
    used = set(c.table.flatten().tolist())
    free = [p for p in range(c.n_pages) if p not in used]
    random.Random(seed).shuffle(free)
    new_table = torch.full((len(lens), -(-max_keep // page)), -1, dtype=torch.int32)
    for b, n in enumerate(lens):
        for j in range(-(-min(n, max(keep[b], 0), max_keep) // page)):
            new_table[b, j] = free.pop()
    for b, j, x in bad_new:
        new_table[b, j] = x
    for b, j, x in bad_old:
        c.table[b, j] = x
    mass = torch.exp(2 * torch.randn((len(lens), hk, pages.max_ctx + 2), generator=c.gen))
    if weigh is not None:
        mass = weigh(mass)
    want_k, want_v = c.k.clone(), c.v.clone()
    kept, new_mass, new_len = torch.full((len(lens), max_keep), -9, dtype=torch.int32), torch.full((len(lens), hk, max_keep), -8.0), []
    table = c.table.cpu()
    for b, n in enumerate(lens):
        rows = R.kept_rows(mass[b], n, min(keep[b], max_keep), n_first, n_recent)
        m = len(rows)
        new_len.append(m)
        kept[b, :m] = torch.tensor(rows, dtype=torch.int32)
        new_mass[b, :, :m] = mass[b][:, rows]
        for j, i in enumerate(rows):
            src, dst = int(table[b, i // page]), int(new_table[b, j // page])
            if 0 <= src < c.n_pages and 0 <= dst < c.n_pages:
                want_k[dst, j % page], want_v[dst, j % page] = c.k[src, i % page], c.v[src, i % page]
    print(hq, hk, d, dtype, page, lens[:5], keep[:5], n_first, n_recent, flush=True)
    got_kept, got_mass = torch.full(kept.shape, -9, dtype=torch.int32, device="cuda"), torch.full(new_mass.shape, -8.0, device="cuda")
    got_len = c.ctx_len if same_len else torch.full((len(lens),), -1, dtype=torch.int32, device="cuda")
    ws = torch.full((B.kvs_workspace_size("evict_paged", c.shape, len(lens), pages.max_ctx),), 255, dtype=torch.uint8, device="cuda")
    gm = mass.cuda()
    B.kvs_evict_paged(c.shape, cache, pages, torch.tensor(keep, dtype=torch.int32, device="cuda"), n_first, n_recent, gm, new_table.cuda(), got_kept, got_len, got_mass, ws)
    assert got_len.tolist() == new_len
    assert torch.equal(got_kept.cpu(), kept)
    assert torch.equal(got_mass.cpu().view(torch.int32), new_mass.view(torch.int32))
    assert torch.equal(_bits(c.k), _bits(want_k)) and torch.equal(_bits(c.v), _bits(want_v))
    assert torch.equal(gm.cpu().view(torch.int32), mass.view(torch.int32))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("hk,d", [(1, 64), (2, 128), (4, 128), (8, 128), (3, 64), (64, 64)])
def test_lengths_and_budgets(hk, d, dtype):
    lens = [0, 1, 2, 15, 16, 17, 33, 100, 257, 300, 300, 300, 300, 300]
    keep = [5, 1, 1, 15, 9, 100, 20, 50, 128, 0, -4, 300, 299, 1]
    _check(2 * hk, hk, d, dtype, 16, lens, keep, 2, 7, seed=hk)
    _check(hk, hk, d, dtype, 64, lens, keep, 0, 0, seed=hk + 1)


def test_protected_rows_that_do_not_fit():
    for first, recent in ((10, 10), (100, 3), (3, 1000), (0, 17), (17, 0), (2 ** 31 - 1, 2 ** 31 - 1)):
        _check(4, 2, 64, BF16, 16, [40, 100, 9, 16], [17, 17, 5, 16], first, recent, seed=first % 100)


def test_ties_zeros_and_odd_weights():
    _check(4, 2, 64, BF16, 16, [300, 500], [100, 77], 1, 4, seed=1, weigh=lambda m: m.round().clamp_max(3))
    _check(4, 2, 64, BF16, 16, [300, 500], [100, 77], 1, 4, seed=2, weigh=lambda m: torch.zeros_like(m))

    def odd(m):
        m = m.clone()
        m[:, :, ::5] = 0.0
        m[:, 0, 1::7] = -0.0
        m[:, :, 3::11] = float("nan")
        m[:, :, 4::13] = float("inf")
        m[:, :, 6::17] = -float("inf")
        m[:, :, 8::19] = -2.5
        m[:, :, 9::23] = 1e-42
        return m
    for keep in ([20, 30], [250, 400], [290, 480]):
        _check(4, 2, 64, BF16, 16, [300, 500], keep, 1, 4, seed=3, weigh=odd)


def test_long_contexts():
    _check(4, 2, 64, BF16, 32, [9000, 12345], [4000, 12000], 4, 100, seed=4)
    _check(8, 4, 128, BF16, 128, [33333], [20000], 4, 1000, seed=5)
    _check(2, 2, 64, BF16, 16, [40000], [17], 4, 1, seed=6, weigh=lambda m: 1 + m * 1e-6)


def test_cut_short_and_without_pages():
    _check(4, 2, 64, BF16, 16, [200, 90], [150, 60], 2, 5, seed=6, max_ctx=120)
    _check(4, 2, 64, BF16, 16, [200, 90], [150, 60], 2, 5, seed=7, max_keep=70)
    _check(4, 2, 64, BF16, 16, [200, 90], [150, 60], 2, 5, seed=8, bad_new=((0, 3, -1), (1, 0, 10 ** 6)), bad_old=((0, 4, -1), (0, 7, 2 ** 31 - 1)))
    _check(4, 2, 64, BF16, 16, [200, 90, 16, 700], [150, 60, 16, 3], 2, 5, seed=9, same_len=True)


def test_many_requests():
    rng = random.Random(3)
    lens = [rng.randrange(0, 200) for _ in range(200)]
    _check(4, 2, 64, BF16, 16, lens, [rng.randrange(0, 100) for _ in lens], 1, 3, seed=10)


def test_lists_alone_and_from_a_graph():
    c = R.Case(4, 2, 64, BF16, 16, [(500, 0), (300, 0)], seed=11)
    cache, pages = c.on()
    mass = torch.rand((2, 2, 500), device="cuda")
    keep = torch.tensor([200, 150], dtype=torch.int32, device="cuda")
    kept = torch.full((2, 200), -9, dtype=torch.int32, device="cuda")
    ws = torch.empty((B.kvs_workspace_size("evict_paged", c.shape, 2, 500),), dtype=torch.uint8, device="cuda")
    k, v = c.k.clone(), c.v.clone()
    call = lambda: B.kvs_evict_paged(c.shape, cache, pages, keep, 4, 20, mass, None, kept, None, None, ws)
    call()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for step in range(4):
        mass.copy_(torch.rand(mass.shape, device="cuda"))
        keep.sub_(9)
        kept.fill_(-9)
        graph.replay()
        torch.cuda.synchronize()
        for b, n in enumerate((500, 300)):
            m = int(keep[b])
            assert kept[b, :m].tolist() == R.kept_rows(mass[b].cpu(), n, m, 4, 20) and (kept[b, m:] == -9).all()
    assert torch.equal(_bits(c.k), _bits(k)) and torch.equal(_bits(c.v), _bits(v))


def test_rows_behind_32_bits():
    n_pages = 6 * 2 ** 30 // (16 * 2 * 128 * 2)
    k, v = (torch.zeros((n_pages, 16, 2, 128), dtype=BF16, device="cuda") for _ in range(2))
    table = torch.tensor([[n_pages - 1, 5, n_pages - 3]], dtype=torch.int32, device="cuda")
    for p in table[0].tolist():
        k[p], v[p] = torch.randn((16, 2, 128), device="cuda").bfloat16(), torch.randn((16, 2, 128), device="cuda").bfloat16()
    sh = B.make_shape(4, 2, 128, B.BF16)
    mass = torch.rand((1, 2, 48), device="cuda")
    to = torch.tensor([[n_pages - 2, n_pages - 4]], dtype=torch.int32, device="cuda")
    kept = torch.zeros((1, 20), dtype=torch.int32, device="cuda")
    ws = torch.empty((B.kvs_workspace_size("evict_paged", sh, 1, 48),), dtype=torch.uint8, device="cuda")
    B.kvs_evict_paged(sh, B.PagedCache(k, v), B.PageTable(table, torch.tensor([48], dtype=torch.int32, device="cuda"), 48), torch.tensor([20], dtype=torch.int32, device="cuda"), 1, 2, mass, to, kept, workspace=ws)
    rows = R.kept_rows(mass[0].cpu(), 48, 20, 1, 2)
    assert kept[0].tolist() == rows
    for j, i in enumerate(rows):
        p, q = int(table[0, i // 16]), int(to[0, j // 16])
        assert torch.equal(k[q, j % 16], k[p, i % 16]) and torch.equal(v[q, j % 16], v[p, i % 16])


@pytest.mark.parametrize("hk,d", [(1, 64), (5, 64)])
@pytest.mark.parametrize("n", [4096, 4097, 8192, 8193, 16384, 16385])
def test_contexts_at_the_ends_of_the_selecting_kernels(hk, d, n):
    _check(hk, hk, d, BF16, 64, [n, n - 1, 7], [700, 333, 5], 3, 100, seed=n + hk)


def test_keys_of_many_parts():
    """More parts than a workgroup has waves, and more keys of one first digit than are asked for early."""
    _check(1, 1, 64, BF16, 256, [140000], [3000], 4, 50, seed=11)
    _check(1, 1, 64, BF16, 256, [140000], [2500], 4, 50, seed=12, weigh=lambda m: m.clamp(1.0, 1.2).mul(64).round())
