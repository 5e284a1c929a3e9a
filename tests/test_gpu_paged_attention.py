"""kvs_attention_paged against attention in 64 bits."""
import random

import pytest
import torch

import paged_ref as R
from paper_2503_16525_amd import binding as B

pytestmark = pytest.mark.gpu

SHAPES = [(28, 4, 128), (32, 8, 128), (7, 1, 128), (40, 1, 128), (6, 6, 64), (4, 4, 128), (64, 2, 64)]
BF16, F32 = torch.bfloat16, torch.float32


def _parts(c):
    return 2 if c.dtype is BF16 and c.n * (c.hq // c.hk) <= 32 * len(c.lens) else 1


def _attend(c, window=0, n_first=0, max_ctx=None, ws_bytes=None, listed=None):
    cache, pages = c.on(max_ctx)
    cu, sel = c.of(listed)
    out, lse = torch.full_like(c.q, 7.0), torch.full((c.n, c.hq), 7.0, device="cuda")
    size = B.kvs_workspace_size("attention_paged", c.shape, len(c.lens), pages.max_ctx, c.n) if ws_bytes is None else ws_bytes
    ws = torch.full((size,), 255, dtype=torch.uint8, device="cuda") if size else None
    B.kvs_attention_paged(c.shape, cache, pages, cu, sel, c.q, c.scale, window, n_first, out, lse, ws)
    return out, lse


def _check(c, what, window=0, n_first=0, bad=None, **kw):
    ref = R.attention(c, window, n_first, bad)
    for ws_bytes in (None, 0):
        name = f"{what}: {c.hq}x{c.hk}x{c.d} {c.dtype} pages of {c.page}, {len(c.lens)} requests of {min(c.lens)} to {max(c.lens)}, {c.n} tokens, window {window} + {n_first}, workspace {ws_bytes}"
        print(name, flush=True)
        out, lse = _attend(c, window, n_first, ws_bytes=ws_bytes, **kw)
        R.check_attention(c, out, lse, ref, _parts(c), name)
        for s in list(range(c.cu[0])) + list(range(c.cu[-1], c.n)):          # places that hold no token
            assert (out[s] == 7).all() and (lse[s] == 7).all(), name


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("hq,hk,d", SHAPES)
def test_single_tokens(hq, hk, d, dtype):
    lens = [0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 100, 129, 500]
    for page in (16, 64):
        _check(R.Case(hq, hk, d, dtype, page, [(n, 1) for n in lens], seed=hq + page), "single tokens")


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("page", [16, 32, 128, 256])
def test_long_single_tokens_in_pieces(page, dtype):
    _check(R.Case(8, 2, 128, dtype, page, [(3001, 1)], seed=page), "long")
    _check(R.Case(8, 2, 128, dtype, page, [(2100, [2099]), (40, 1), (0, 1), (1500, [7, 1499]), (5000, 1)], seed=page), "ragged")


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("hq,hk,d", [(28, 4, 128), (8, 8, 64), (32, 8, 128), (3, 1, 64), (40, 1, 128)])
def test_chunks(hq, hk, d, dtype):
    """The last tokens of their requests: whole prompts, chunks, none, more than the context holds."""
    _check(R.Case(hq, hk, d, dtype, 32, [(300, 300)], seed=1), "whole prompt")
    _check(R.Case(hq, hk, d, dtype, 16, [(260, 33), (1, 1), (20, 0), (90, 90), (0, 3), (333, 100), (5, 9), (64, 64)], seed=2, places=(3, 5)), "ragged")
    _check(R.Case(hq, hk, d, dtype, 128, [(900, 130)], seed=3), "chunk")


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("hq,hk,d", [(28, 4, 128), (8, 8, 64), (3, 1, 64)])
def test_selected_tokens(hq, hk, d, dtype):
    rng = random.Random(hq)
    pick = lambda n, k: sorted(rng.sample(range(n), k))
    _check(R.Case(hq, hk, d, dtype, 32, [(700, pick(700, 90))], seed=1), "one request")
    _check(R.Case(hq, hk, d, dtype, 16, [(260, pick(260, 33)), (1, [0]), (0, []), (90, pick(90, 1)), (333, pick(333, 100))], seed=2), "ragged")
    # any order, the same twice, none, past the context
    _check(R.Case(hq, hk, d, dtype, 64, [(300, [299, 0, 5, 5, 299, -1, 77, 100000, -1000]), (50, [-1, -1]), (0, [0, -1, 3])], seed=3, places=(1, 2)), "any order")


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("window,n_first", [(1, 0), (5, 1), (31, 4), (32, 0), (33, 33), (64, 100), (100, 4), (1000, 7), (2 ** 31 - 1, 2 ** 31 - 1)])
def test_windows(window, n_first, dtype):
    _check(R.Case(8, 2, 128, dtype, 16, [(700, 1), (3, 1), (0, 1), (200, 1), (64, 1)], seed=window % 1000), "single tokens", window, n_first)
    _check(R.Case(8, 2, 128, dtype, 32, [(700, 60), (3, 3), (200, 200), (64, 0)], seed=window % 1000 + 1), "chunks", window, n_first)
    _check(R.Case(6, 3, 64, dtype, 64, [(700, [0, 1, 40, 350, 351, 699, -1, 800]), (90, [89, 3, 3])], seed=3), "selected", window, n_first)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_windows_of_long_contexts(dtype):
    _check(R.Case(8, 2, 128, dtype, 16, [(6000, 1), (9000, 1)], seed=5), "long window", 2500, 40)
    _check(R.Case(4, 1, 128, dtype, 16, [(5000, 300)], seed=6), "long chunk", 1111, 70)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("scale", [0.125, -0.7, 0.0])
def test_scales_of_the_scores(scale, dtype):
    _check(R.Case(4, 4, 64, dtype, 16, [(130, [0, 64, 129])], scale=scale, seed=7), f"scale {scale}")
    _check(R.Case(4, 2, 128, dtype, 16, [(300, 300)], scale=scale, seed=8), f"scale {scale}")


def test_more_requests_than_lanes():
    rng = random.Random(0)
    lens = [rng.randrange(0, 90) for _ in range(300)]
    _check(R.Case(8, 2, 64, BF16, 16, [(n, 1) for n in lens], seed=9), "300 requests")
    _check(R.Case(8, 2, 128, BF16, 16, [(n, min(n, rng.choice([0, 0, 1, 2, 9, 40]))) for n in lens], seed=10, places=(2, 70)), "300 ragged requests")


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d", [64, 128])
def test_what_a_row_does_not_see_does_not_reach_it(d, dtype):
    """Infinities and NaN in rows of a context that only later tokens see, and in such that a window leaves out."""
    odd = [33, 40, 41, 64, 95, 96, 210]

    def change(y, b, is_v):
        y = y.clone()
        for j, i in enumerate(odd):
            if i < y.shape[0]:
                y[i, j % 2, ::7] = [float("nan"), float("inf"), -float("inf")][(j + is_v) % 3]
        return y

    clean = R.Case(4, 2, d, dtype, 16, [(220, [0, 20, 32, 32]), (100, [10, 32]), (34, [5])], seed=4)
    c = R.Case(4, 2, d, dtype, 16, [(220, [0, 20, 32, 32]), (100, [10, 32]), (34, [5])], seed=4, change=change)
    ref = R.attention(c)
    assert torch.isfinite(ref[0]).all()
    for a, b in zip(ref[:3], R.attention(clean)[:3]):
        assert torch.equal(a, b)
    out, lse = _attend(c)
    R.check_attention(c, out, lse, ref, _parts(c), "later rows")
    # a window from 98 on, beside the first 30
    c = R.Case(4, 2, d, dtype, 16, [(205, [150, 200, 204])], seed=4, change=change)
    ref = R.attention(c, 53, 30)
    out, lse = _attend(c, 53, 30)
    R.check_attention(c, out, lse, ref, _parts(c), "a window")
    # V alone: the channels of the rows that see it
    def change_v(y, b, is_v):
        y = y.clone()
        if is_v:
            y[33, 1, 5] = float("nan")
            y[60, 0, 9] = float("inf")
        return y
    c = R.Case(4, 2, d, dtype, 16, [(100, [20, 32, 33, 45, 59, 60, 61, 99])], seed=4, change=change_v)
    out, lse = _attend(c)
    assert torch.isfinite(lse).all()
    broken = torch.zeros_like(out, dtype=torch.bool)
    broken[2:, 2:, 5] = True
    broken[5:, :2, 9] = True
    assert torch.equal(~torch.isfinite(out), broken)
    assert torch.isnan(out[2:, 2:, 5]).all() and (out[5:, :2, 9] == torch.inf).all()
    c0 = R.Case(4, 2, d, dtype, 16, [(100, [20, 32, 33, 45, 59, 60, 61, 99])], seed=4)
    ref = R.attention(c0)
    out = torch.where(broken, ref[0].to(out.dtype), out)
    R.check_attention(c0, out, lse, ref, _parts(c0), "single channels")


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_entries_that_name_no_page(dtype):
    """Their rows are not seen, wherever they stand: also where nothing else is left."""
    for window, n_first in ((0, 0), (70, 20)):
        c = R.Case(8, 2, 128, dtype, 16, [(300, [0, 20, 31, 32, 47, 48, 200, 299]), (33, [31, 32]), (16, [15])], seed=6)
        bad = [torch.zeros((n,), dtype=torch.bool, device="cuda") for n in c.lens]
        for b, p, x in ((0, 2, -1), (0, 7, c.n_pages), (0, 18, -2 ** 31), (1, 2, 2 ** 31 - 1), (2, 0, -5)):
            c.table[b, p] = x
            bad[b][16 * p:16 * p + 16] = True
        _check(c, "no page", window, n_first, bad)


def test_a_length_beyond_what_the_host_promised():
    """max_ctx rows are taken, or as many as the table names; a negative length is none."""
    c = R.Case(4, 2, 64, BF16, 16, [(200, [50, 199]), (90, [89])], seed=8)
    short = R.Case(4, 2, 64, BF16, 16, [(200, [50, 199]), (90, [89])], seed=8)
    short.lens = [120, 90]
    short.slots[0] = short.slots[0][:120]
    ref = R.attention(short)
    out, lse = _attend(c, max_ctx=120)
    R.check_attention(short, out, lse, ref, _parts(c), "max_ctx")
    c.ctx_len.copy_(torch.tensor([2 ** 31 - 1, -5], dtype=torch.int32))
    c.lens = [208, 0]
    c.table[0, 12] = c.table[0, 3]                            # a page that has numbers in all of its rows
    c.slots[0] = c.table[0, torch.arange(208, device="cuda") // 16].long() * 16 + torch.arange(208, device="cuda") % 16
    out, lse = _attend(c, max_ctx=5000)
    R.check_attention(c, out, lse, R.attention(c), _parts(c), "the table's width")


def test_large_scores_and_falling_ones():
    """Scores that rise and fall by hundreds from tile to tile, and rows that one key dominates."""
    def change(y, b, is_v):
        y = y.clone()
        if not is_v:
            y[::37] *= 60
        return y
    for dtype in (BF16, F32):
        _check(R.Case(2, 1, 64, dtype, 16, [(700, [0, 15, 16, 300, 699])], seed=4, change=change, scale=1.0), "large scores")
        _check(R.Case(4, 1, 128, dtype, 16, [(1500, 200)], seed=5, change=change, scale=1.0), "large scores")


def test_any_workspace_will_do():
    c = R.Case(4, 1, 128, BF16, 32, [(5000, [10, 4000, 4999])], seed=17)
    ref = R.attention(c)
    full = B.kvs_workspace_size("attention_paged", c.shape, 1, 5000, 3)
    for size in (0, 256, 20000, 60001, full // 2, full):
        out, lse = _attend(c, ws_bytes=size)
        R.check_attention(c, out, lse, ref, _parts(c), f"workspace of {size}")


def test_no_log_sum_exps():
    c = R.Case(8, 2, 128, BF16, 16, [(2500, 1), (40, 1)], seed=19)
    cache, pages = c.on()
    out = torch.empty_like(c.q)
    B.kvs_attention_paged(c.shape, cache, pages, None, None, c.q, c.scale, 0, 0, out)
    R.check_attention(c, out, None, R.attention(c), _parts(c), "no lse")


def test_a_pool_behind_32_bits():
    """Pages 6 GB into a pool."""
    c = R.Case(4, 2, 128, BF16, 16, [(100, 40), (33, 1)], seed=21)
    n_pages = 6 * 2 ** 30 // (16 * 2 * 128 * 2)
    big = [torch.zeros((n_pages, 16, 2, 128), dtype=BF16, device="cuda") for _ in range(2)]
    far = n_pages - c.n_pages
    for x, y in zip(big, (c.k, c.v)):
        x[far:] = y
    table = c.table + far
    out, lse = torch.empty_like(c.q), torch.empty((c.n, c.hq), device="cuda")
    B.kvs_attention_paged(c.shape, B.PagedCache(*big), B.PageTable(table, c.ctx_len, 100), c.cu_new, None, c.q, c.scale, 0, 0, out, lse)
    R.check_attention(c, out, lse, R.attention(c), _parts(c), "far pages")


def test_replays_from_a_graph_with_other_contexts():
    """A decode step captured once, replayed while the contexts grow and change their pages."""
    c = R.Case(8, 2, 128, BF16, 16, [(1000, 1), (37, 1), (0, 1), (2500, 1)], seed=23, width=200, spare=40)
    cache, pages = c.on(3200)
    ws = [torch.empty((B.kvs_workspace_size("attention_paged", c.shape, 4, 3200, 4),), dtype=torch.uint8, device="cuda") for _ in range(2)]
    outs, lses = [torch.empty_like(c.q) for _ in range(2)], [torch.empty((4, 8), device="cuda") for _ in range(2)]
    call = lambda i: B.kvs_attention_paged(c.shape, cache, pages, None, None, c.q, c.scale, 0, 0, outs[i], lses[i], ws[i])
    call(1)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(1)
    nan = torch.isnan(c.k)
    c.k[nan], c.v[nan] = 0.5, 0.25
    for step in range(4):
        graph.replay()
        torch.cuda.synchronize()
        outs[0].fill_(9.0)
        call(0)
        torch.cuda.synchronize()
        assert torch.equal(outs[0], outs[1]) and torch.equal(lses[0], lses[1]), step
        assert torch.equal(torch.isinf(lses[0]).all(1).cpu(), c.ctx_len.cpu() == 0)
        c.ctx_len.add_(torch.tensor([1, 1, 17, -300], dtype=torch.int32, device="cuda"))
        c.table[2, :4] = c.table[0, 5:9]
        c.table[1].copy_(c.table[1].roll(1) if step == 2 else c.table[1])
        c.q.mul_(-1.25)


def test_another_stream():
    c = R.Case(8, 2, 128, BF16, 16, [(1000, 1), (2500, 1)], seed=25)
    cache, pages = c.on()
    ref = R.attention(c)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    out, lse = torch.empty_like(c.q), torch.empty((2, 8), device="cuda")
    ws = torch.empty((B.kvs_workspace_size("attention_paged", c.shape, 2, 2500, 2),), dtype=torch.uint8, device="cuda")
    B.kvs_attention_paged(c.shape, cache, pages, None, None, c.q, c.scale, 0, 0, out, lse, ws, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    R.check_attention(c, out, lse, ref, _parts(c), "stream")


def test_equal_calls_give_equal_bits():
    c = R.Case(32, 8, 128, BF16, 16, [(3000, 500), (2000, 1), (700, 700)], seed=27)
    first = _attend(c)
    for _ in range(3):
        for a, b in zip(first, _attend(c)):
            assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("hq,hk,d", [(8, 2, 128), (28, 4, 128), (6, 6, 64)])
def test_one_request_of_many_tokens_among_many_of_one(hq, hk, d, dtype):
    """Few rows a request on average, but not in all: some come in several blocks."""
    many = 32 * 40 * hk // hq - 40
    reqs = [(30 + 7 * i, 1) for i in range(39)]
    reqs.insert(20, (many + 100, many))
    _check(R.Case(hq, hk, d, dtype, 16, reqs, seed=31), "skewed")
    _check(R.Case(hq, hk, d, dtype, 16, reqs, seed=32), "skewed", 50, 5)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d,tokens", [(64, 40), (128, 40), (128, 300)])
def test_a_query_that_is_no_number_reaches_its_row_only(d, tokens, dtype):
    c = R.Case(4, 2, d, dtype, 16, [(400, tokens), (50, 1)], seed=33)
    ref = R.attention(c)
    c.q[7, 2, 5], c.q[tokens, 0, 0] = float("nan"), float("inf")
    out, lse = _attend(c)
    broken = torch.zeros((c.n, 4), dtype=torch.bool, device="cuda")
    broken[7, 2] = broken[tokens, 0] = True
    assert torch.isnan(out[broken]).all() and torch.isnan(lse[broken]).all()
    out[broken], lse[broken] = ref[0][broken].to(dtype), ref[1][broken].float()
    R.check_attention(c, out, lse, ref, _parts(c), "broken queries")
