"""The kernel of kvs_attention_paged for many rows a key (256 a workgroup), against attention in 64 bits.  Its estimate takes it for calls of some size only, so
each case below says how it goes there, and the host's choice is compared with that before the call: small ones through the second build of the
library, with a number of pieces that the case names, and calls that the shipped library sends there by itself."""
import random

import pytest
import torch

import paged_many as M
import paged_ref as R
from paper_2503_16525_amd import binding as B
from test_gpu_paged_attention import _attend

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


def _there(lib, c, pieces, dealt, window=0, n_first=0, max_ctx=None, ws_bytes=None):
    """The host's choice for the call that _attend makes of c."""
    cu, sel = c.of()
    longest = max(max(c.lens), 1) if max_ctx is None else max_ctx
    taken = M.choice(lib, c.shape, c.page, len(c.lens), min(longest, c.width * c.page), c.n, cu is not None, sel is not None, c.scale, window, n_first, ws_bytes, c.n_pages)
    assert taken == (True, pieces, dealt), taken


def _run(c, pieces, what, window=0, n_first=0, bad=None, ref=None, dealt=False, force=True):
    """One call with so many pieces -> out, lse, checked"""
    ref = R.attention(c, window, n_first, bad) if ref is None else ref
    name = f"{what}: {c.hq}x{c.hk}, pages of {c.page}, {len(c.lens)} requests of {min(c.lens)} to {max(c.lens)}, {c.n} tokens, window {window} + {n_first}, {pieces} pieces"
    print(name, flush=True)
    with M.forced(pieces if force else 0) as lib:
        _there(lib, c, pieces, dealt, window, n_first)
        if force:
            out, lse = _attend(c, window, n_first)
    if not force:                                            # (the shipped library)
        out, lse = _attend(c, window, n_first)
    R.check_attention(c, out, lse, ref, 1, name)
    for s in list(range(c.cu[0])) + list(range(c.cu[-1], c.n)):          # places that hold no token
        assert (out[s] == 7).all() and (lse[s] == 7).all(), name
    return out, lse


@pytest.mark.parametrize("hq,hk", [(28, 4), (32, 8), (4, 4), (40, 1), (64, 2)])
def test_lengths_around_tiles_and_steps(hq, hk):
    for n in (1, 31, 32, 33, 63, 64, 65, 95, 96, 97, 127, 160, 161, 257):
        page = [16, 64, 256][n % 3]
        _run(R.Case(hq, hk, 128, BF16, page, [(n + 64, n)], seed=n), 1, "behind some")
        _run(R.Case(hq, hk, 128, BF16, page, [(n, n)], seed=n), 1, "a prompt")
    _run(R.Case(hq, hk, 128, BF16, 16, [(n, n) for n in (300, 1, 65, 250, 33, 0, 129)], seed=3, places=(2, 3)), 1, "prompts")


def test_single_tokens():
    _run(R.Case(32, 8, 128, BF16, 16, [(n, 1) for n in (0, 1, 16, 33, 64, 500, 1111)], seed=1), 1, "one token each")
    _run(R.Case(28, 4, 128, BF16, 64, [(3000, 1)], seed=2), 5, "one token")


@pytest.mark.parametrize("pieces", [1, 2, 7])
def test_chunks_behind_long_contexts(pieces):
    for n, m in ((2000, 200), (4100, 65), (3333, 777), (5000, 256)):
        _run(R.Case(8, 2, 128, BF16, 16, [(n, m)], seed=n), pieces, "chunk")
    _run(R.Case(28, 4, 128, BF16, 32, [(1500, 300), (800, 5), (0, 0), (2900, 100), (77, 77), (40, 60)], seed=5, places=(1, 4)), pieces, "ragged")


@pytest.mark.parametrize("window,n_first", [(1, 0), (5, 1), (31, 4), (32, 0), (33, 33), (64, 100), (100, 4), (500, 64), (1000, 7), (2 ** 31 - 1, 2 ** 31 - 1)])
def test_windows(window, n_first):
    rng = random.Random(window)
    chunk = R.Case(8, 2, 128, BF16, 16, [(1200, 400)], seed=window % 1000)
    ragged = R.Case(28, 4, 128, BF16, 64, [(700, 700), (300, 40), (33, 33)], seed=window % 1000)
    selected = R.Case(16, 2, 128, BF16, 32, [(900, sorted(rng.sample(range(900), 80))), (300, [299, 3, 3, -1, 500] * 9)], seed=2)
    for pieces in (1, 2, 3):
        if pieces == 1 or window >= 500:                     # (pieces of fewer than eight tiles are not made)
            _run(chunk, pieces, "chunk", window, n_first)
        if pieces == 1 or (pieces == 2 and window >= 500):
            _run(ragged, pieces, "ragged", window, n_first)
        _run(selected, pieces, "selected", window, n_first)


@pytest.mark.parametrize("pieces", [1, 4])
def test_selected_tokens(pieces):
    rng = random.Random(7)
    pick = lambda n, k: sorted(rng.sample(range(n), k))
    _run(R.Case(32, 8, 128, BF16, 16, [(3000, pick(3000, 333))], seed=1), pieces, "one request")
    _run(R.Case(28, 4, 128, BF16, 32, [(1700, pick(1700, 190)), (1, [0]), (0, [0, 2, -1]), (90, pick(90, 1)), (999, pick(999, 100))], seed=2, places=(3, 4)), pieces, "ragged")
    _run(R.Case(16, 2, 128, BF16, 64, [(1500, [1499, 0, -1, 70, 10 ** 9, 33] * 12), (50, [-1] * 40), (0, [0, -1, 3])], seed=3), pieces, "any order")


@pytest.mark.parametrize("pieces", [1, 3])
@pytest.mark.parametrize("step,by", [(37, 60.0), (200, 300.0), (5, 20.0)])
def test_references_move(step, by, pieces):
    """Rows whose scores rise by hundreds behind their first tile, and rows that a few keys dominate."""
    def change(y, b, is_v):
        y = y.clone()
        if not is_v:
            y[40::step] *= by
        return y
    _run(R.Case(4, 1, 128, BF16, 16, [(1500, 200)], seed=5, change=change, scale=1.0), pieces, f"every {step}th key times {by}")
    _run(R.Case(4, 1, 128, BF16, 16, [(1700, 900)], seed=6, change=change, scale=1.0), pieces, f"every {step}th key times {by}", 900, 3)
    if pieces == 1:
        _run(R.Case(4, 1, 128, BF16, 16, [(900, 900)], seed=6, change=change, scale=1.0), pieces, f"every {step}th key times {by}", 100, 3)


@pytest.mark.parametrize("plateau", [54, 84, 114])
@pytest.mark.parametrize("pieces", [1, 3])
def test_a_reference_that_moves_keeps_what_came_before(plateau, pieces):
    """The first tile's scores are 0, those of the next thousand keys `plateau` powers of two above, so that their sum may have grown to just below what
    moves a reference; then one key stands above all of them by a little or a lot, and counts for as much as they do together or
    for more.  (Whole scores, which bf16 holds.)"""
    n, high = 1100, 1050

    def levels(rise):
        level = torch.zeros((n,))
        level[32:1032] = plateau
        level[high] = plateau + rise
        return level

    for rise in (8, 10, 11, 12, 13, 14, 15, 17, 20, 33, 64, 100):
        def change(y, b, is_v):
            if is_v:
                y = y.abs() + 1                              # V of one sign, so that nothing that is lost cancels
                y[high] = -y[high]
                return y
            k = torch.zeros_like(y)
            k[:, 0, 0] = (levels(rise) / 64).floor()         # times 64
            k[:, 0, 1] = levels(rise) % 64
            return k
        c = R.Case(4, 1, 128, BF16, 16, [(n, 40)], seed=3, change=change, scale=0.6931471805599453)
        c.q[:] = 0
        c.q[:, :, 0], c.q[:, :, 1] = 64, 1
        _run(c, pieces, f"a plateau of {plateau}, then {rise} more")


@pytest.mark.parametrize("first,second", [(60, 63), (63, 67), (63, 130), (120, 124), (123, 126), (123, 127), (123, 130), (123, 133), (200, 203), (127, 123)])
def test_pieces_whose_first_tiles_lie_far_apart(first, second):
    """Two pieces.  The first one's scores begin at 0 and rise to `first` powers of two in one key; the second one's begin with a tile of
    one key at `second`: each counts by its largest score, wherever its reference stands."""
    n, half = 1100, 576                                      # 18 tiles of 32 keys each

    def change(y, b, is_v):
        if is_v:
            y = y.abs() + 1                                  # V of one sign, times 8 where the scores are lower
            y[200] *= 8
            return y
        level = torch.zeros((n,))
        level[200], level[half + 3] = first, second
        k = torch.zeros_like(y)
        k[:, 0, 0], k[:, 0, 1] = (level / 64).floor(), level % 64
        return k
    c = R.Case(4, 1, 128, BF16, 16, [(n, 20)], seed=8, change=change, scale=0.6931471805599453)
    c.q[:] = 0
    c.q[:, :, 0], c.q[:, :, 1] = 64, 1
    _run(c, 2, f"{first} beside {second}")


@pytest.mark.parametrize("pieces", [0, 1, 3])
@pytest.mark.parametrize("power", [-100, -90, -70, 60, 100])
def test_small_and_large_values(power, pieces):
    """V of a magnitude far from 1, by this kernel and (0 pieces) by the one that takes such a call otherwise: what comes out is as near as ever, relative to
    what goes in (compared after a multiplication by the power of two, so that no absolute floor helps)."""
    def level(y, b, is_v):
        if is_v:
            return y * 2.0 ** power
        y = y.clone()
        y[100:700] *= 6.0                                    # references that move, in some rows often
        return y
    for scale, change in ((None, lambda y, b, is_v: y * 2.0 ** power if is_v else y), (1.0, level)):
        c = R.Case(8, 2, 128, BF16, 16, [(900, 300), (40, 40)], seed=power % 17, change=change, scale=scale)
        out, lse, mag, dots = R.attention(c)
        with M.forced(pieces) as lib:
            if pieces:
                _there(lib, c, pieces, False)
            got, got_lse = _attend(c)
        R.check_attention(c, got.double() * 2.0 ** -power, got_lse, (out * 2.0 ** -power, lse, mag * 2.0 ** -power, dots), 1, f"V of 2^{power}")


@pytest.mark.parametrize("window,n_first,pieces", [(0, 0, 1), (0, 0, 3), (48, 33, 1), (89, 33, 1)])
def test_what_a_row_does_not_see_does_not_reach_it(window, n_first, pieces):
    odd = [33, 40, 41, 64, 95, 96, 500, 511, 512, 700]

    def change(y, b, is_v):
        y = y.clone()
        for j, i in enumerate(odd):
            if i < y.shape[0]:
                y[i, j % 2, ::7] = [float("nan"), float("inf"), -float("inf")][(j + is_v) % 3]
        return y

    # tokens in front of all of them, and those behind 600 of which a window covers none
    front = list(range(33)) * 4
    reqs = {0: [(800, front), (790, front)], 48: [(800, front), (34, [5] * 60), (650, list(range(560, 650)))], 89: [(800, list(range(601, 690)))]}[window]
    clean, c = (R.Case(8, 2, 128, BF16, 16, reqs, seed=4, change=f) for f in (None, change))
    ref = R.attention(c, window, n_first)
    assert torch.isfinite(ref[0]).all()
    for a, b in zip(ref[:3], R.attention(clean, window, n_first)[:3]):
        assert torch.equal(a, b)
    _run(c, pieces, "not seen", window, n_first, ref=ref)


@pytest.mark.parametrize("pieces", [1, 3])
def test_a_v_that_is_no_number(pieces):
    def change(y, b, is_v):
        y = y.clone()
        if is_v:
            y[133, 1, 5] = float("nan")
            y[260, 0, 9] = float("inf")
        return y
    c, clean = (R.Case(8, 2, 128, BF16, 16, [(900, 900)], seed=4, change=f) for f in (change, None))
    with M.forced(pieces) as lib:
        _there(lib, c, pieces, False)
        out, lse = _attend(c)
    broken = torch.zeros_like(out, dtype=torch.bool)
    broken[133:, 4:, 5] = True
    broken[260:, :4, 9] = True
    assert torch.equal(~torch.isfinite(out), broken) and torch.isfinite(lse).all()
    assert torch.isnan(out[133:, 4:, 5]).all() and (out[260:, :4, 9] == torch.inf).all()
    R.check_attention(clean, torch.where(broken, R.attention(clean)[0].to(BF16), out), lse, R.attention(clean), 1, "single channels")


def test_a_v_that_only_the_last_piece_holds():
    def change(y, b, is_v):
        y = y.clone()
        if is_v:
            y[2990, 0, 0] = float("inf")
        return y
    c, clean = (R.Case(4, 1, 128, BF16, 16, [(3000, 100)], seed=9, change=f) for f in (change, None))
    ref = R.attention(clean)
    for pieces in (2, 11):
        with M.forced(pieces) as lib:
            _there(lib, c, pieces, False)
            out, lse = _attend(c)
        assert (out[90:, :, 0] == torch.inf).all() and torch.isfinite(out[:90]).all() and torch.isfinite(out[:, :, 1:]).all()
        out[90:, :, 0] = ref[0][90:, :, 0].to(BF16)
        R.check_attention(clean, out, lse, ref, 1, "pieces")


def test_queries_that_are_no_numbers():
    c = R.Case(8, 2, 128, BF16, 16, [(700, 300), (40, 40)], seed=14)
    ref = R.attention(c)
    good = c.q.clone()
    c.q[17, 3, 5], c.q[200, 0, 0], c.q[320, 7, 127] = float("nan"), float("nan"), float("nan")
    for pieces in (1, 2):
        with M.forced(pieces) as lib:
            _there(lib, c, pieces, False)
            out, lse = _attend(c)
        for s, h in ((17, 3), (200, 0), (320, 7)):
            assert torch.isnan(out[s, h]).all() and torch.isnan(lse[s, h])
            out[s, h], lse[s, h] = ref[0][s, h].to(BF16), ref[1][s, h].float()
        R.check_attention(c, out, lse, ref, 1, "broken queries")
    c.q.copy_(good)


@pytest.mark.parametrize("window,n_first,pieces", [(0, 0, 1), (0, 0, 3), (70, 20, 1), (600, 20, 2)])
def test_entries_that_name_no_page(window, n_first, pieces):
    c = R.Case(8, 2, 128, BF16, 16, [(900, 300), (33, [31, 32] * 40), (16, [15] * 9)], seed=6)
    bad = [torch.zeros((n,), dtype=torch.bool, device="cuda") for n in c.lens]
    for b, p, x in ((0, 2, -1), (0, 7, c.n_pages), (0, 45, -2 ** 31), (1, 2, 2 ** 31 - 1), (2, 0, -5)):
        c.table[b, p] = x
        bad[b][16 * p:16 * p + 16] = True
    _run(c, pieces, "no page", window, n_first, bad)


def test_workspaces_that_hold_fewer_pieces():
    """What fits is taken, to the byte: in the shipped library's own choice, more pieces need more, and a workspace of nothing another kernel."""
    c = R.Case(28, 4, 128, BF16, 32, [(6000, 300)], seed=17)
    ref = R.attention(c)
    full = B.kvs_workspace_size("attention_paged", c.shape, 1, 6000, 300)
    rows = 300 * 28 * (128 * 4 + 16)                         # a piece's sums
    seen = set()
    for size in (0, 255, 256, 2048, rows, 2 * rows + 256, 2 * rows + 4096, 4 * rows + 4096, 5 * rows + 4096, 6 * rows + 4096, full):
        with M.forced(0) as lib:
            seen.add(M.choice(lib, c.shape, 32, 1, 6000, 300, ws_bytes=size)[:2])
        out, lse = _attend(c, ws_bytes=size)
        R.check_attention(c, out, lse, ref, 1, f"workspace of {size}")
    assert {x for x in seen if x[0]} >= {(True, 4), (True, 5), (True, 6), (True, 7)}, seen
    two = R.Case(8, 2, 128, BF16, 32, [(3000, 150)], seed=18)
    ref = R.attention(two)
    rows = 150 * 8 * (128 * 4 + 16)
    for pieces in (2, 5):
        least = 256 + pieces * rows                          # a word for each of a few workgroups, and the sums
        with M.forced(pieces) as lib:
            _there(lib, two, pieces, False, ws_bytes=least)
            assert not M.choice(lib, two.shape, 32, 1, 3000, 150, ws_bytes=least - 1)[0]
            out, lse = _attend(two, ws_bytes=least)
        R.check_attention(two, out, lse, ref, 1, f"{pieces} pieces in {least} bytes")


def test_more_requests_than_lanes():
    rng = random.Random(1)
    lens = [rng.randrange(0, 200) for _ in range(130)]
    _run(R.Case(16, 2, 128, BF16, 16, [(n, min(n, rng.choice([0, 17, 40, 200]))) for n in lens], seed=10, places=(2, 70)), 1, "130 ragged requests")
    lens = [rng.randrange(300, 600) for _ in range(70)]
    _run(R.Case(8, 2, 128, BF16, 16, [(n, rng.choice([0, 1, 17, 70])) for n in lens], seed=11, places=(2, 70)), 2, "70 in pieces")


@pytest.mark.parametrize("pieces", [1, 3])
def test_replays_from_a_graph_with_other_contexts(pieces):
    """Two captured calls that share a workspace, replayed in turn, as contexts grow and shrink."""
    c = R.Case(8, 2, 128, BF16, 16, [(1000, 60), (370, 100)], seed=23, width=80, rest=0.25, spare=20)
    with M.forced(pieces) as lib:
        _there(lib, c, pieces, False, max_ctx=1200)
        cache, pages = c.on(1200)
        ws = [torch.empty((B.kvs_workspace_size("attention_paged", c.shape, 2, 1200, 160),), dtype=torch.uint8, device="cuda") for _ in range(2)]
        outs, lses = [torch.empty_like(c.q) for _ in range(3)], [torch.empty((160, 8), device="cuda") for _ in range(3)]
        call = lambda i: B.kvs_attention_paged(c.shape, cache, pages, c.cu_new, None, c.q, c.scale, 0, 0, outs[i], lses[i], ws[min(i, 1)])
        call(1)
        graphs = []
        for i in (1, 2):
            graphs.append(torch.cuda.CUDAGraph())
            with torch.cuda.graph(graphs[-1]):
                call(i)
        for step in range(4):
            for o in outs:
                o.fill_(9.0)
            graphs[0].replay()
            graphs[1].replay()
            torch.cuda.synchronize()
            call(0)
            torch.cuda.synchronize()
            for i in (1, 2):
                assert torch.equal(outs[0], outs[i]) and torch.equal(lses[0], lses[i]), step
            c.ctx_len.add_(torch.tensor([-50, 20], dtype=torch.int32, device="cuda"))
            c.cu_new[1] += 7
            c.q.mul_(-1.25)


@pytest.mark.parametrize("pieces", [1, 2])
def test_a_pool_behind_32_bits(pieces):
    c = R.Case(4, 2, 128, BF16, 16, [(600, 140), (33, 20)], seed=21)
    n_pages = 6 * 2 ** 30 // (16 * 2 * 128 * 2)
    big = [torch.zeros((n_pages, 16, 2, 128), dtype=BF16, device="cuda") for _ in range(2)]
    far = n_pages - c.n_pages
    for x, y in zip(big, (c.k, c.v)):
        x[far:] = y
    out, lse = torch.empty_like(c.q), torch.empty((c.n, c.hq), device="cuda")
    with M.forced(pieces) as lib:
        _there(lib, c, pieces, False)
        ws = torch.empty((B.kvs_workspace_size("attention_paged", c.shape, 2, 600, 160),), dtype=torch.uint8, device="cuda")
        B.kvs_attention_paged(c.shape, B.PagedCache(*big), B.PageTable(c.table + far, c.ctx_len, 600), c.cu_new, None, c.q, c.scale, 0, 0, out, lse, ws)
    R.check_attention(c, out, lse, R.attention(c), 1, "far pages")


@pytest.mark.parametrize("hq,hk,n,window,n_first", [(64, 2, 1100, 0, 0), (64, 2, 1301, 200, 3), (32, 8, 2100, 300, 40), (40, 1, 1700, 0, 0), (64, 4, 1100, 33, 0)])
def test_more_row_tiles_than_compute_units(hq, hk, n, window, n_first):
    """One request's: each workgroup takes several, of which the first ones hold a V that only later tokens may multiply."""
    def change(y, b, is_v):
        y = y.clone()
        if is_v:
            y[n - 1, 0, 7] = float("nan")
        return y
    _run(R.Case(hq, hk, 128, BF16, 32, [(n, list(range(n - 1)) + [0])], seed=n, change=change), 1, "dealt", window, n_first, dealt=True)
    _run(R.Case(hq, hk, 128, BF16, 16, [(n + 77, n)], seed=n + 1), 1, "dealt chunk", window, n_first, dealt=True)


@pytest.mark.parametrize("hq,hk,n,m,window,n_first,pieces,dealt", [
    (32, 8, 16000, 256, 0, 0, 8, False), (28, 4, 6000, 300, 0, 0, 7, False), (32, 8, 3000, 1000, 0, 0, 2, False), (32, 8, 2000, 2000, 0, 0, 1, False),
    (64, 2, 2000, 2000, 0, 0, 1, True), (64, 2, 2000, 2000, 700, 3, 1, True), (28, 4, 6000, 6000, 4000, 4, 1, True)])
def test_calls_that_the_shipped_library_sends_there(hq, hk, n, m, window, n_first, pieces, dealt):
    """One request's last rows; then the same numbers of picked rows, whose choice is the same without a window."""
    _run(R.Case(hq, hk, 128, BF16, 16, [(n, m)], seed=n), pieces, "shipped", window, n_first, dealt=dealt, force=False)
    if not window and m < n:
        _run(R.Case(hq, hk, 128, BF16, 64, [(n, sorted(random.Random(n).sample(range(n), m)))], seed=n + 1), pieces, "shipped, selected", dealt=dealt, force=False)


def test_equal_calls_give_equal_bits():
    for pieces, dealt, c in ((1, False, R.Case(8, 2, 128, BF16, 16, [(1500, 400), (300, 20)], seed=2)), (4, False, R.Case(8, 2, 128, BF16, 16, [(1500, 400), (300, 20)], seed=2)),
                             (1, True, R.Case(64, 2, 128, BF16, 16, [(1200, 1100)], seed=2))):
        with M.forced(pieces) as lib:
            _there(lib, c, pieces, dealt)
            first = _attend(c)
            for _ in range(4):
                assert all(torch.equal(a, b) for a, b in zip(first, _attend(c)))
