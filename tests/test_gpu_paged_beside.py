"""The calls on a cache in pages where everything that they read and write lies side by side in one allocation, touching but not overlapping, and where
they may write over what they read: accepted, and right."""
import pytest
import torch

import paged_many as M
import paged_ref as R
from paper_2503_16525_amd import binding as B
from test_gpu_paged_attention import _parts

pytestmark = pytest.mark.gpu


class Lot:
    """Slices of one allocation, one behind the other (tensors of 256 bytes and more begin at multiples of 256)"""

    def __init__(self, size):
        self.all, self.at = torch.zeros((size,), dtype=torch.uint8, device="cuda"), 0

    def take(self, like):
        n = like.numel() * like.element_size()
        part = self.all[self.at:self.at + n].view(like.dtype).view(like.shape)
        part.copy_(like)
        self.at += n
        return part


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_side_by_side(dtype):
    hq, hk, d, page, taken = 8, 2, 128, 16, 128
    c = R.Case(hq, hk, d, dtype, page, [(taken, 64), (64, 64), (96, 32), (32, 32)], seed=1, rest=0.0, spare=9, width=8)
    lot = Lot(1 << 24)
    batch, i32 = 4, dict(dtype=torch.int32, device="cuda")
    c.k, c.v = lot.take(c.k), lot.take(c.v)
    k_new, v_new = (lot.take(torch.randn((c.n, hk, d), generator=c.gen).to(dtype)) for _ in range(2))
    c.q = lot.take(c.q)
    out = lot.take(torch.zeros_like(c.q))
    lse = lot.take(torch.zeros((c.n, hq), device="cuda"))
    mass, mass_out = (lot.take(torch.rand((batch, hk, taken), generator=c.gen)) for _ in range(2))
    new_mass, kept = lot.take(torch.zeros((batch, hk, 32))), lot.take(torch.zeros((batch, 32), dtype=torch.int32))
    c.table = lot.take(c.table)
    used = set(c.table.flatten().tolist())
    free = [i for i in range(c.n_pages) if i not in used]
    new_table = lot.take(torch.tensor(free[:8], **i32).view(batch, 2))
    keep, new_len, c.ctx_len = lot.take(torch.tensor([32, 17, 5, 0], **i32)), lot.take(torch.zeros((batch,), **i32)), lot.take(c.ctx_len)
    c.cu_new = lot.take(c.cu_new)
    lot.at = (lot.at + 255) // 256 * 256
    cache, pages = B.PagedCache(c.k, c.v), B.PageTable(c.table, c.ctx_len, taken)
    B.kvs_store_paged(c.shape, cache, pages, c.cu_new, None, k_new, v_new, mass)
    for b in range(batch):
        rows = c.slots[b][c.pos[b]].cuda()
        assert torch.equal(c.k.view(-1, hk, d)[rows], k_new[c.cu[b]:c.cu[b + 1]]) and torch.equal(c.v.view(-1, hk, d)[rows], v_new[c.cu[b]:c.cu[b + 1]])
        assert not mass[b, :, c.pos[b]].any()
    ref = R.attention(c)
    ws = lot.all[lot.at:lot.at + B.kvs_workspace_size("attention_paged", c.shape, batch, taken, c.n)]
    B.kvs_attention_paged(c.shape, cache, pages, c.cu_new, None, c.q, c.scale, 0, 0, out, lse, ws)
    R.check_attention(c, out, lse, ref, _parts(c), "side by side")
    want = R.mass(c, lse, mass, 0.5)
    ws = lot.all[lot.at:lot.at + B.kvs_workspace_size("mass_paged", c.shape, batch, taken, c.n)]
    B.kvs_mass_paged(c.shape, cache, pages, c.cu_new, None, c.q, lse, c.scale, 0, 0, 0.5, mass, mass_out, ws)
    R.check_mass(c, mass_out, want, lse, "side by side")
    B.kvs_mass_paged(c.shape, cache, pages, c.cu_new, None, c.q, lse, c.scale, 0, 0, 0.5, mass, mass, ws)
    for b, n in enumerate(c.lens):
        assert torch.equal(mass[b, :, :n], mass_out[b, :, :n])
    rows = [R.kept_rows(mass[b].cpu(), n, int(keep[b]), 2, 3) for b, n in enumerate(c.lens)]
    before = c.k.clone()
    ws = lot.all[lot.at:lot.at + B.kvs_workspace_size("evict_paged", c.shape, batch, taken)]
    for lengths in (new_len, c.ctx_len):                     # beside the old lengths, then over them
        B.kvs_evict_paged(c.shape, cache, pages, keep, 2, 3, mass, new_table, kept, lengths, new_mass, ws)
        for b, want_rows in enumerate(rows):
            m = len(want_rows)
            assert int(lengths[b]) == m and kept[b, :m].tolist() == want_rows
            assert torch.equal(new_mass[b, :, :m], mass[b][:, want_rows])
            for j, i in enumerate(want_rows):
                assert torch.equal(c.k[int(new_table[b, j // page]), j % page], before[int(c.table[b, i // page]), i % page])


@pytest.mark.parametrize("dtype,pieces", [(torch.bfloat16, None), (torch.bfloat16, 1), (torch.bfloat16, 2), (torch.float32, None)])
def test_places_that_hold_no_token(dtype, pieces):
    """Before the first and behind the last request's tokens: NaN and infinities in them reach nothing, and nothing of theirs is written.  By the kernels of
    few and of many rows a request, and (pieces) by attention's for many rows a key."""
    for reqs in ([(600, 300), (64, 5), (0, 0), (33, 33)], [(600, 1), (64, 2), (33, 1), (40, 3)]):
        c = R.Case(8, 2, 128, dtype, 16, reqs, seed=6, places=(70, 90))
        ref = R.attention(c)
        lse = torch.nan_to_num(ref[1], nan=0.0).float()
        old = torch.rand((len(reqs), 2, 600), generator=c.gen).cuda()
        want = R.mass(c, lse, old, 1.0)
        k_new, v_new = (torch.randn((c.n, 2, 128), generator=c.gen).to(dtype).cuda() for _ in range(2))
        for x in (c.q, k_new, v_new, lse):
            x[:c.cu[0]], x[c.cu[-1]:] = float("nan"), float("inf")
        cache, pages = c.on()
        out, got_lse = torch.full_like(c.q, 7.0), torch.full((c.n, 8), 7.0, device="cuda")
        ws = torch.empty((max(B.kvs_workspace_size(x, c.shape, len(reqs), 600, c.n) for x in ("attention_paged", "mass_paged")),), dtype=torch.uint8, device="cuda")
        with M.forced(pieces or 0) as lib:
            assert not pieces or M.choice(lib, c.shape, 16, len(reqs), 600, c.n)[:2] == (True, pieces)
            B.kvs_attention_paged(c.shape, cache, pages, c.cu_new, None, c.q, c.scale, 0, 0, out, got_lse, ws)
        R.check_attention(c, out, got_lse, ref, 1 if pieces else _parts(c), "places")
        for s in (slice(0, c.cu[0]), slice(c.cu[-1], c.n)):
            assert (out[s] == 7).all() and (got_lse[s] == 7).all()
        got = old.clone()
        B.kvs_mass_paged(c.shape, cache, pages, c.cu_new, None, c.q, lse, c.scale, 0, 0, 1.0, got, got, ws)
        R.check_mass(c, got, want, lse[c.cu[0]:c.cu[-1]], "places")
        B.kvs_store_paged(c.shape, cache, pages, c.cu_new, None, k_new, v_new)
        for b in range(len(reqs)):
            rows = c.slots[b].cuda()
            assert torch.isfinite(c.k.view(-1, 2, 128)[rows]).all()
            assert torch.equal(c.v.view(-1, 2, 128)[rows[c.pos[b]]], v_new[c.cu[b]:c.cu[b + 1]])
