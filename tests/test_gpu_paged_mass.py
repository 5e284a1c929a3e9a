"""kvs_mass_paged against column sums in 64 bits."""
import random

import pytest
import torch

import paged_ref as R
from paper_2503_16525_amd import binding as B

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


def _check(c, what, window=0, n_first=0, bad=None, decay=1.0, max_ctx=None):
    cache, pages = c.on(max_ctx)
    cu, sel = c.of()
    ref = R.attention(c, window, n_first, bad)
    lse = torch.where(torch.isnan(ref[1]), torch.zeros_like(ref[1]), ref[1]).float()
    stride = pages.max_ctx + 5
    old = torch.rand((len(c.lens), c.hk, stride), generator=c.gen).cuda()
    want = R.mass(c, lse, old, decay, window, n_first, bad)
    for ws_bytes in (None, 0):
        for in_place in (True, False):
            name = f"{what}: {c.hq}x{c.hk}x{c.d} {c.dtype} pages of {c.page}, {len(c.lens)} requests of {min(c.lens)} to {max(c.lens)}, {c.n} tokens, window {window} + {n_first}, workspace {ws_bytes}"
            print(name, flush=True)
            size = B.kvs_workspace_size("mass_paged", c.shape, len(c.lens), pages.max_ctx, c.n) if ws_bytes is None else ws_bytes
            ws = torch.full((size,), 255, dtype=torch.uint8, device="cuda") if size else None
            before = old.clone()
            got = before if in_place else torch.full_like(old, 5.0)
            B.kvs_mass_paged(c.shape, cache, pages, cu, sel, c.q, lse, c.scale, window, n_first, decay, before, got, ws)
            R.check_mass(c, got, want, lse, name)
            for b, n in enumerate(c.lens):                       # behind the contexts
                assert torch.equal(got[b, :, n:], old[b, :, n:] if in_place else torch.full_like(old[b, :, n:], 5.0)), name
            if not in_place:
                assert torch.equal(before, old)
    got = torch.full_like(old, 5.0)
    B.kvs_mass_paged(c.shape, cache, pages, cu, sel, c.q, lse, c.scale, window, n_first, decay, None, got)
    R.check_mass(c, got, (want[0] - decay * old.double(), want[1], want[2]), lse, what + ", from nothing")
    return got


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("hq,hk,d", [(28, 4, 128), (32, 8, 128), (40, 1, 128), (6, 6, 64), (64, 2, 64)])
def test_single_tokens(hq, hk, d, dtype):
    lens = [0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 100, 129, 255, 256, 257, 700]
    for page in (16, 128):
        _check(R.Case(hq, hk, d, dtype, page, [(n, 1) for n in lens], seed=hq + page), "single tokens", decay=0.75)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("hq,hk,d", [(28, 4, 128), (8, 8, 64), (3, 1, 64), (40, 1, 128)])
def test_chunks_and_selected_tokens(hq, hk, d, dtype):
    rng = random.Random(hq)
    got = _check(R.Case(hq, hk, d, dtype, 32, [(300, 300)], seed=1), "whole prompt")
    assert torch.allclose(got[0, :, :300].sum(-1), torch.full((hk,), 300.0 * hq / hk, device="cuda"), rtol=1e-4)      # every row's weights add up to 1
    _check(R.Case(hq, hk, d, dtype, 16, [(260, 33), (1, 1), (20, 0), (90, 90), (0, 3), (333, 100), (5, 9)], seed=2, places=(3, 5)), "ragged", decay=0.0)
    _check(R.Case(hq, hk, d, dtype, 64, [(300, [299, 0, 5, 5, 299, -1, 77, 100000, -1000]), (50, [-1, -1]), (700, sorted(rng.sample(range(700), 90)))], seed=3), "any order")


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("window,n_first", [(1, 0), (31, 4), (33, 33), (100, 4), (300, 400), (2 ** 31 - 1, 2 ** 31 - 1)])
def test_windows(window, n_first, dtype):
    _check(R.Case(8, 2, 128, dtype, 16, [(1000, 1), (3, 1), (0, 1), (200, 1), (64, 1)], seed=window % 1000), "single tokens", window, n_first)
    _check(R.Case(8, 2, 128, dtype, 32, [(1000, 60), (3, 3), (400, 400), (64, 0)], seed=window % 1000 + 1), "chunks", window, n_first)
    _check(R.Case(6, 3, 64, dtype, 64, [(700, [0, 1, 40, 350, 351, 699, -1, 800]), (90, [89, 3, 3])], seed=3), "selected", window, n_first)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_rows_in_pieces(dtype):
    """Chunks of many rows over few keys, whose sums are joined."""
    c = R.Case(16, 2, 128, dtype, 16, [(900, 700)], seed=4)
    assert B.kvs_workspace_size("mass_paged", c.shape, 1, 900, 700) > 256
    _check(c, "pieces", decay=0.5)
    _check(R.Case(16, 2, 128, dtype, 16, [(900, 700), (50, 40), (0, 0), (600, 600)], seed=5), "ragged pieces", 100, 3)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("scale", [-0.7, 0.0])
def test_scales(scale, dtype):
    _check(R.Case(4, 2, 64, dtype, 16, [(130, 130), (40, 1)], scale=scale, seed=7), f"scale {scale}")


def test_more_requests_than_lanes():
    rng = random.Random(0)
    lens = [rng.randrange(0, 90) for _ in range(150)]
    _check(R.Case(8, 2, 64, BF16, 16, [(n, 1) for n in lens], seed=9), "150 requests")
    _check(R.Case(8, 2, 128, BF16, 16, [(n, min(n, rng.choice([0, 0, 1, 2, 9, 40]))) for n in lens], seed=10, places=(2, 70)), "150 ragged requests")


def test_entries_that_name_no_page():
    for dtype in (BF16, F32):
        c = R.Case(8, 2, 128, dtype, 16, [(300, [0, 20, 31, 32, 47, 48, 200, 299]), (33, [31, 32]), (16, [15])], seed=6)
        bad = [torch.zeros((n,), dtype=torch.bool, device="cuda") for n in c.lens]
        for b, p, x in ((0, 2, -1), (0, 7, c.n_pages), (0, 18, -2 ** 31), (1, 2, 2 ** 31 - 1), (2, 0, -5)):
            c.table[b, p] = x
            bad[b][16 * p:16 * p + 16] = True
        _check(c, "no page", bad=bad, decay=0.5)


def test_keys_that_a_row_does_not_see_may_hold_anything():
    def change(y, b, is_v):
        y = y.clone()
        y[40:60] = float("nan")
        return y
    _check(R.Case(4, 2, 64, BF16, 16, [(100, [0, 20, 39])], seed=4, change=change), "later rows")
    _check(R.Case(4, 2, 64, BF16, 16, [(100, [90, 95, 99])], seed=4, change=change), "a window", 30, 40)


def test_a_pool_behind_32_bits():
    c = R.Case(4, 2, 128, BF16, 16, [(100, 40), (33, 1)], seed=21)
    n_pages = 6 * 2 ** 30 // (16 * 2 * 128 * 2)
    big = torch.zeros((n_pages, 16, 2, 128), dtype=BF16, device="cuda")
    far = n_pages - c.n_pages
    big[far:] = c.k
    lse = R.attention(c)[1].float()
    old = torch.rand((2, 2, 100), device="cuda")
    got = torch.empty_like(old)
    B.kvs_mass_paged(c.shape, B.PagedCache(big, big), B.PageTable(c.table + far, c.ctx_len, 100), c.cu_new, None, c.q, lse, c.scale, 0, 0, 0.9, old, got)
    R.check_mass(c, got, R.mass(c, lse, old, 0.9), lse, "far pages")


def test_replays_from_a_graph():
    c = R.Case(8, 2, 128, BF16, 16, [(400, 1), (37, 1), (0, 1)], seed=23, width=40, rest=0.25, spare=40)
    cache, pages = c.on(640)
    lse = torch.full((3, 8), 6.0, device="cuda")
    mass = [torch.zeros((3, 2, 640), device="cuda") for _ in range(2)]
    call = lambda i: B.kvs_mass_paged(c.shape, cache, pages, None, None, c.q, lse, c.scale, 0, 0, 0.9, mass[i], mass[i])
    call(0)
    call(1)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(1)
    for step in range(4):
        c.ctx_len.add_(5)
        graph.replay()
        call(0)
        torch.cuda.synchronize()
        assert torch.equal(*mass), step
        c.q.mul_(-1.1)
    assert (mass[0][0, :, :400] > 0).all() and (mass[0][:, :, 600:] == 0).all()
    assert (mass[0][2] == 0).all()                              # its table names no page


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("hq,hk,d", [(8, 2, 128), (28, 4, 128), (6, 6, 64)])
def test_one_request_of_many_tokens_among_many_of_one(hq, hk, d, dtype):
    """Few rows a request on average, but not in all: some come in several blocks."""
    many = 32 * 40 * hk // hq - 40
    reqs = [(30 + 7 * i, 1) for i in range(39)]
    reqs.insert(20, (many + 100, many))
    _check(R.Case(hq, hk, d, dtype, 16, reqs, seed=31), "skewed")
    _check(R.Case(hq, hk, d, dtype, 16, reqs, seed=32), "skewed", 50, 5)
