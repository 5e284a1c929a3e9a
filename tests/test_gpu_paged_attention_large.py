"""kvs_attention_paged where many rows share their keys (bf16, 128 channels: 256 rows a workgroup), against attention in 64 bits."""
import random

import pytest
import torch

import paged_ref as R
from paper_2503_16525_amd import binding as B
from test_gpu_paged_attention import _attend, _check

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


@pytest.mark.parametrize("hq,hk", [(28, 4), (32, 8), (4, 4), (40, 1), (64, 2)])
@pytest.mark.parametrize("page", [16, 64, 256])
def test_lengths_around_tiles_and_steps(hq, hk, page):
    grp = hq // hk
    for n in (1, 31, 32, 33, 63, 64, 65, 95, 96, 97, 127, 160, 161, 257):
        _check(R.Case(hq, hk, 128, BF16, page, [(n + 64, max(n, 128 // grp + 1))], seed=n), "one request")
    _check(R.Case(hq, hk, 128, BF16, page, [(n, n) for n in (300, 1, 65, 250, 33, 0, 129)], seed=page, places=(2, 3)), "prompts")


def test_chunks_behind_long_contexts():
    for n, m in ((2000, 200), (4100, 65), (3333, 1111), (5000, 256)):
        _check(R.Case(8, 2, 128, BF16, 16, [(n, m)], seed=n), "chunk")
    _check(R.Case(28, 4, 128, BF16, 32, [(1500, 300), (800, 5), (0, 0), (2900, 100), (77, 77)], seed=5), "ragged")


@pytest.mark.parametrize("window,n_first", [(1, 0), (5, 1), (31, 4), (32, 0), (33, 33), (64, 100), (100, 4), (500, 64), (1000, 7), (2 ** 31 - 1, 2 ** 31 - 1)])
def test_windows(window, n_first):
    _check(R.Case(8, 2, 128, BF16, 16, [(1200, 400)], seed=window % 1000), "chunk", window, n_first)
    _check(R.Case(28, 4, 128, BF16, 64, [(700, 700), (300, 40), (33, 33)], seed=window % 1000), "ragged", window, n_first)
    rng = random.Random(window)
    _check(R.Case(16, 2, 128, BF16, 32, [(900, sorted(rng.sample(range(900), 80))), (300, [299, 3, 3, -1, 500] * 9)], seed=2), "selected", window, n_first)


def test_selected_tokens():
    rng = random.Random(7)
    pick = lambda n, k: sorted(rng.sample(range(n), k))
    _check(R.Case(32, 8, 128, BF16, 16, [(3000, pick(3000, 333))], seed=1), "one request")
    _check(R.Case(28, 4, 128, BF16, 32, [(700, pick(700, 190)), (1, [0]), (0, [0, 2, -1]), (90, pick(90, 1)), (999, pick(999, 100))], seed=2, places=(3, 4)), "ragged")
    _check(R.Case(16, 2, 128, BF16, 64, [(500, [499, 0, -1, 70, 10 ** 9, 33] * 12), (50, [-1] * 40), (0, [0, -1, 3])], seed=3), "any order")


def test_references_move():
    """Rows whose scores rise by hundreds behind their first tile, in one tile or over many, and rows that a few keys dominate."""
    for step, by in ((37, 60.0), (200, 300.0), (5, 20.0)):
        def change(y, b, is_v):
            y = y.clone()
            if not is_v:
                y[40::step] *= by
            return y
        _check(R.Case(4, 1, 128, BF16, 16, [(1500, 200)], seed=5, change=change, scale=1.0), f"every {step}th key times {by}")
        _check(R.Case(4, 1, 128, BF16, 16, [(900, 900)], seed=6, change=change, scale=1.0), f"every {step}th key times {by}", 100, 3)

    def rising(y, b, is_v):
        return y if is_v else y * torch.linspace(0, 60, y.shape[0])[:, None, None]
    _check(R.Case(4, 1, 128, BF16, 16, [(1500, 200)], seed=7, change=rising, scale=0.5), "rising")


def test_what_a_row_does_not_see_does_not_reach_it():
    odd = [33, 40, 41, 64, 95, 96, 500, 511, 512, 700]

    def change(y, b, is_v):
        y = y.clone()
        for j, i in enumerate(odd):
            if i < y.shape[0]:
                y[i, j % 2, ::7] = [float("nan"), float("inf"), -float("inf")][(j + is_v) % 3]
        return y

    # tokens in front of all of them, and those behind 600 of which a window covers none
    front = list(range(33)) * 4
    for reqs, window, n_first in (([(800, front)], 0, 0), ([(800, list(range(601, 690)))], 89, 33), ([(800, front), (34, [5] * 60), (650, list(range(560, 650)))], 48, 33)):
        clean, c = (R.Case(8, 2, 128, BF16, 16, reqs, seed=4, change=f) for f in (None, change))
        ref = R.attention(c, window, n_first)
        assert torch.isfinite(ref[0]).all()
        for a, b in zip(ref[:3], R.attention(clean, window, n_first)[:3]):
            assert torch.equal(a, b)
        for ws_bytes in (None, 0):
            out, lse = _attend(c, window, n_first, ws_bytes=ws_bytes)
            R.check_attention(c, out, lse, ref, 1, f"{reqs[0][0]} {window}")

    def change_v(y, b, is_v):
        y = y.clone()
        if is_v:
            y[133, 1, 5] = float("nan")
            y[260, 0, 9] = float("inf")
        return y
    c, clean = (R.Case(8, 2, 128, BF16, 16, [(900, 900)], seed=4, change=f) for f in (change_v, None))
    out, lse = _attend(c)
    broken = torch.zeros_like(out, dtype=torch.bool)
    broken[133:, 4:, 5] = True
    broken[260:, :4, 9] = True
    assert torch.equal(~torch.isfinite(out), broken) and torch.isfinite(lse).all()
    assert torch.isnan(out[133:, 4:, 5]).all() and (out[260:, :4, 9] == torch.inf).all()
    ref = R.attention(clean)
    R.check_attention(clean, torch.where(broken, ref[0].to(BF16), out), lse, ref, 1, "single channels")


def test_entries_that_name_no_page():
    for window, n_first in ((0, 0), (70, 20)):
        c = R.Case(8, 2, 128, BF16, 16, [(900, 300), (33, [31, 32] * 40), (16, [15] * 9)], seed=6)
        bad = [torch.zeros((n,), dtype=torch.bool, device="cuda") for n in c.lens]
        for b, p, x in ((0, 2, -1), (0, 7, c.n_pages), (0, 45, -2 ** 31), (1, 2, 2 ** 31 - 1), (2, 0, -5)):
            c.table[b, p] = x
            bad[b][16 * p:16 * p + 16] = True
        _check(c, "no page", window, n_first, bad)


def test_pieces_with_what_they_cannot_multiply():
    """A chunk that is cut, in whose last piece stands a V that only the last tokens see."""
    def change(y, b, is_v):
        y = y.clone()
        if is_v:
            y[2990, 0, 0] = float("inf")
        return y
    c, clean = (R.Case(4, 1, 128, BF16, 16, [(3000, 100)], seed=9, change=f) for f in (change, None))
    out, lse = _attend(c)
    assert (out[90:, :, 0] == torch.inf).all() and torch.isfinite(out[:90]).all() and torch.isfinite(out[:, :, 1:]).all()
    ref = R.attention(clean)
    out[90:, :, 0] = ref[0][90:, :, 0].to(BF16)
    R.check_attention(clean, out, lse, ref, 1, "pieces")


def test_any_workspace_will_do():
    c = R.Case(8, 2, 128, BF16, 32, [(3000, 150)], seed=17)
    ref = R.attention(c)
    full = B.kvs_workspace_size("attention_paged", c.shape, 1, 3000, 150)
    for size in (0, 256, 100000, 2 * 10 ** 6 + 1, full // 2, full):
        out, lse = _attend(c, ws_bytes=size)
        R.check_attention(c, out, lse, ref, 1, f"workspace of {size}")


def test_more_requests_than_lanes():
    rng = random.Random(1)
    lens = [rng.randrange(0, 200) for _ in range(130)]
    _check(R.Case(16, 2, 128, BF16, 16, [(n, min(n, rng.choice([0, 17, 40, 200]))) for n in lens], seed=10, places=(2, 70)), "130 ragged requests")


def test_replays_from_a_graph_with_other_contexts():
    c = R.Case(8, 2, 128, BF16, 16, [(1000, 60), (370, 100)], seed=23, width=80, rest=0.25, spare=20)
    cache, pages = c.on(1200)
    ws = [torch.empty((B.kvs_workspace_size("attention_paged", c.shape, 2, 1200, 160),), dtype=torch.uint8, device="cuda") for _ in range(2)]
    outs, lses = [torch.empty_like(c.q) for _ in range(2)], [torch.empty((160, 8), device="cuda") for _ in range(2)]
    call = lambda i: B.kvs_attention_paged(c.shape, cache, pages, c.cu_new, None, c.q, c.scale, 0, 0, outs[i], lses[i], ws[i])
    call(1)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(1)
    for step in range(4):
        graph.replay()
        torch.cuda.synchronize()
        outs[0].fill_(9.0)
        call(0)
        torch.cuda.synchronize()
        assert torch.equal(outs[0], outs[1]) and torch.equal(lses[0], lses[1]), step
        c.ctx_len.add_(torch.tensor([-50, 20], dtype=torch.int32, device="cuda"))
        c.cu_new[1] += 7
        c.q.mul_(-1.25)


def test_a_pool_behind_32_bits():
    c = R.Case(4, 2, 128, BF16, 16, [(300, 140), (33, 20)], seed=21)
    n_pages = 6 * 2 ** 30 // (16 * 2 * 128 * 2)
    big = [torch.zeros((n_pages, 16, 2, 128), dtype=BF16, device="cuda") for _ in range(2)]
    far = n_pages - c.n_pages
    for x, y in zip(big, (c.k, c.v)):
        x[far:] = y
    out, lse = torch.empty_like(c.q), torch.empty((c.n, c.hq), device="cuda")
    ws = torch.empty((B.kvs_workspace_size("attention_paged", c.shape, 2, 300, 160),), dtype=torch.uint8, device="cuda")
    B.kvs_attention_paged(c.shape, B.PagedCache(*big), B.PageTable(c.table + far, c.ctx_len, 300), c.cu_new, None, c.q, c.scale, 0, 0, out, lse, ws)
    R.check_attention(c, out, lse, R.attention(c), 1, "far pages")


@pytest.mark.parametrize("hq,hk,n,window,n_first", [(64, 2, 1100, 0, 0), (64, 2, 1301, 200, 3), (32, 8, 2100, 300, 40), (40, 1, 1700, 0, 0), (64, 4, 1100, 33, 0)])
def test_more_row_tiles_than_compute_units(hq, hk, n, window, n_first):
    """One request's: each workgroup takes several, of which the first ones hold a V that only later tokens may multiply."""
    def change(y, b, is_v):
        y = y.clone()
        if is_v:
            y[n - 1, 0, 7] = float("nan")
        return y
    c = R.Case(hq, hk, 128, BF16, 32, [(n, list(range(n - 1)) + [0])], seed=n, change=change)
    _check(c, "dealt", window, n_first)
    _check(R.Case(hq, hk, 128, BF16, 16, [(n + 77, n)], seed=n + 1), "dealt chunk", window, n_first)
