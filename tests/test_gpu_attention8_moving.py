"""kvs_attention_kv8 over contexts that are widened to more bytes than the last-level cache holds: the softmax reference moves where a row's sum of
weights outgrows it, under factors for every 16 keys.  Rows in the order of shares, of a workgroup a tile and of a queue; every
row against 64 bits, log-sum-exps with them."""
import pytest
import torch

import kv8_torch as T
from paper_2503_16525_amd import binding as B

pytestmark = pytest.mark.gpu

# query heads, KV heads, contexts and the tokens of each: K and V of the longest above 192 MiB in bf16, and 384 tiles of 256 rows or more
LAUNCHES = {
    "shares": (64, 8, [49200], [1600]),
    "a list in order": (64, 8, [49200] + [2000] * 8, [1600] + [128] * 8),
    "a workgroup a tile": (64, 64, [6208], [3800]),
    "a queue": (64, 64, [6208, 6200], [1900, 1900]),
}


def _check(launch, code, block, change, q_of=None, want_lse=True, plain=False):
    hq, hk, ln, ks = LAUNCHES[launch]
    sh = B.make_shape(hq, hk, 128, B.BF16)
    off = [0]
    for n in ln[:-1]:
        off.append(off[-1] + -(-n // block) * block)
    n_rows, grp, n0 = off[-1] + ln[-1], hq // hk, ln[0]
    gen = torch.Generator().manual_seed(7)
    q = torch.randn((sum(ks), hq, 128), generator=gen)
    q = (q / q.norm(dim=-1, keepdim=True)).to(torch.bfloat16).cuda()
    u = q[7, ::grp].float()                                # a direction for each KV head
    if q_of is not None:
        q = q_of(q, u, grp)
    cache = T.normal_cache(n_rows, hk, 128, block, code, 3, lambda x, t: change(x[:n0], u) if t == 0 and change else None)
    # evenly, the last token among them
    pos = torch.cat([n - 1 - torch.arange(k - 1, -1, -1) * (n // k) for n, k in zip(ln, ks)]).to(torch.int32).cuda()
    cu = [sum(ks[:b]) for b in range(len(ln) + 1)]
    size = B.kvs_workspace_size("attention_kv8", sh, len(ln), n_rows, cu[-1])
    ws = torch.full((size,), 255, dtype=torch.uint8, device="cuda")
    out, lse = torch.full_like(q, 7.0), torch.full((cu[-1], hq), 7.0, device="cuda") if want_lse else None
    print(f"{launch}, {code}/{block}, lse {want_lse}", flush=True)
    B.kvs_attention_kv8(sh, cache, off, ln, cu, q, pos, 1.0, out, lse, ws)
    assert bool((ws[size - 4096:] != 255).any()), "the contexts were not widened"
    want, want_lse_, mag, dots, most = T.attention(q, pos, cache, off, ln, cu, 1.0)
    # a weight and the output rounded to bf16, 2^-8 each; scores and sums in fp32; what a key adds is lost below 2^-65 of the output
    fp32 = (132 * dots + 64 + max(ln)) * 2.0 ** -24
    tol = 2.0 ** -8 * (2 * mag + want.abs()) + 2 * fp32 * mag + max(ln) * (2.0 ** -64 * most[None, :, None] + 2.0 ** -65)
    over = (out.double() - want).abs() - tol
    assert bool((over <= 0).all()), float(over.max())
    if want_lse:
        assert bool(((lse.double() - want_lse_).abs() <= fp32 + 2.0 ** -22 * want_lse_.abs()).all())
    if plain:
        assert T.off_by(out, want) <= 1.57 * T.off_by(want.to(torch.bfloat16), want)      # a weight's and the output's rounding: 1.41; V's too: 1.73
    return sh, cache, off, ln, cu, q, pos, ws, out, lse


def _all_alike(q, u, grp):
    return u.repeat_interleave(grp, 0).to(torch.bfloat16).expand_as(q).contiguous()


@pytest.mark.parametrize("launch", list(LAUNCHES))
@pytest.mark.parametrize("code,block", [("e4m3", 32), ("int8", 16)])
def test_plain(launch, code, block):
    _check(launch, code, block, None, plain=True)
    _check(launch, code, block, None, want_lse=False, plain=True)


@pytest.mark.parametrize("launch", list(LAUNCHES))
@pytest.mark.parametrize("code,block,want_lse", [("e4m3", 16, True), ("int8", 64, True), ("e4m3", 128, False)])
def test_reference_moves(launch, code, block, want_lse):
    """In steps of 90 above the key before, in every row; in one row alone; in the last row's own tile; past what fp32 holds."""
    def steps(x, u):
        n = x.shape[0]
        for i, at in enumerate((40, 1000, 1017, n // 2, n - n // 5)):
            x[at] = u * 90 * (i + 1)

    def one_row(x, u):
        x[x.shape[0] // 2] = u * 400

    def last(x, u):
        x[-17] = u * 500

    def jump(x, u):
        x[x.shape[0] // 2] = u * 3000

    def first_far_below(x, u):                             # the first tile at -200, the next key at 150
        x[:32] = u * -200
        x[40] = u * 150
    _check(launch, code, block, steps, _all_alike, want_lse)
    _check(launch, code, block, one_row, None, want_lse)
    _check(launch, code, block, last, _all_alike, want_lse)
    _check(launch, code, block, jump, _all_alike, want_lse)
    _check(launch, code, block, first_far_below, _all_alike, want_lse)


@pytest.mark.parametrize("launch", list(LAUNCHES))
def test_references_too_far_to_move(launch):
    """Logits beyond 2^16 (in powers of two): the tile's exact maxima."""
    def far(x, u):
        x[x.shape[0] // 3] = u * 30000
        x[x.shape[0] // 2] = u * 90000
    _check(launch, "int8", 32, far, _all_alike)


def test_a_broken_block_reaches_the_rows_that_see_it():
    sh, cache, off, ln, cu, q, pos, ws, out, lse = _check("shares", "e4m3", 32, None)
    for scale in (cache.k_scale, cache.v_scale):
        was = scale[1200, 3].clone()
        scale[1200, 3] = float("nan")
        got, got_lse = torch.full_like(q, 7.0), torch.full_like(lse, 7.0)
        B.kvs_attention_kv8(sh, cache, off, ln, cu, q, pos, 1.0, got, got_lse, ws)
        scale[1200, 3] = was
        broken = torch.zeros_like(lse, dtype=torch.bool)
        broken[:, 24:32] = (pos >= 1200 * 32)[:, None]
        assert torch.equal(got_lse.isnan(), broken) and torch.equal(got.isnan(), broken[..., None].expand_as(got))
        # (workgroups that see it take their rows' exact maxima: the others' rows are the same, theirs rounded otherwise)
        fine = ~broken
        assert bool(((got[fine].float() - out[fine].float()).abs() <= 2.0 ** -6 * cache.v_scale.max() * 448).all())


def test_replays_from_a_graph():
    def rise(x, u):
        x[3000] = u * 250
    call = _check("a queue", "int8", 32, rise, _all_alike)
    sh, cache, off, ln, cu, q, pos, ws, out, lse = call
    outs, lses = torch.empty_like(out), torch.empty_like(lse)
    ws2 = torch.empty_like(ws)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        B.kvs_attention_kv8(sh, cache, off, ln, cu, q, pos, 1.0, outs, lses, ws2)
    for i in range(3):
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(outs, out) and torch.equal(lses, lse), i
        q.mul_(0.9)
        cache.v_scale.mul_(1.1)
        B.kvs_attention_kv8(sh, cache, off, ln, cu, q, pos, 1.0, out, lse, ws)
