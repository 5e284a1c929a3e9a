"""The calls on a cache in pages as a serving loop makes them: prompts in chunks over shared pages, decode steps, contexts cut down, and
the loop's captured form."""
import pytest
import torch

import paged_ref as R
from paper_2503_16525_amd import binding as B

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


class Loop:
    """Requests with a page table, and beside the pool what each of its rows has to be (`k`, `v`: lists of rows a request)."""

    def __init__(self, hq, hk, d, dtype, page, batch, width, pages, seed=0):
        self.hq, self.hk, self.d, self.dtype, self.page, self.width = hq, hk, d, dtype, page, width
        self.shape = B.make_shape(hq, hk, d, B.BF16 if dtype is BF16 else B.F32)
        self.cache = B.PagedCache(*(torch.full((pages, page, hk, d), float("nan"), dtype=dtype, device="cuda") for _ in range(2)))
        self.free = list(range(pages))
        self.gen = torch.Generator().manual_seed(seed)
        self.table = torch.full((batch, width), -1, dtype=torch.int32, device="cuda")
        self.ctx_len = torch.zeros((batch,), dtype=torch.int32, device="cuda")
        self.pages = B.PageTable(self.table, self.ctx_len, width * page)
        self.mass = torch.zeros((batch, hk, width * page), device="cuda")
        self.k, self.v = ([torch.zeros((0, hk, d), device="cuda", dtype=dtype) for _ in range(batch)] for _ in range(2))
        self.want_mass = [torch.zeros((hk, 0), dtype=torch.float64, device="cuda") for _ in range(batch)]
        self.scale = d ** -0.5

    def grow(self, b, n):
        """room for rows up to n, and the new length"""
        for i in range(int((self.table[b] >= 0).sum()), -(-n // self.page)):
            self.table[b, i] = self.free.pop(0)
        self.ctx_len[b] = n

    def rand(self, *shape):
        return torch.randn(shape, generator=self.gen).to(self.dtype).cuda()

    def step(self, new, window=0, n_first=0):
        """`new` tokens of each request: stored, attending, counted; everything compared"""
        n, batch = sum(new), len(new)
        cu = [0]
        for m in new:
            cu.append(cu[-1] + m)
        k, v, q = self.rand(n, self.hk, self.d), self.rand(n, self.hk, self.d), self.rand(n, self.hq, self.d)
        for b, m in enumerate(new):
            self.grow(b, self.k[b].shape[0] + m)
            self.k[b], self.v[b] = torch.cat((self.k[b], k[cu[b]:cu[b + 1]])), torch.cat((self.v[b], v[cu[b]:cu[b + 1]]))
        cut = None if new == [1] * batch else torch.tensor(cu, dtype=torch.int32, device="cuda")
        out, lse = torch.full_like(q, 7.0), torch.full((n, self.hq), 7.0, device="cuda")
        ws = [torch.empty((B.kvs_workspace_size(c, self.shape, batch, self.pages.max_ctx, n),), dtype=torch.uint8, device="cuda") for c in ("attention_paged", "mass_paged")]
        B.kvs_store_paged(self.shape, self.cache, self.pages, cut, None, k, v, self.mass)
        B.kvs_attention_paged(self.shape, self.cache, self.pages, cut, None, q, self.scale, window, n_first, out, lse, ws[0])
        B.kvs_mass_paged(self.shape, self.cache, self.pages, cut, None, q, lse, self.scale, window, n_first, 1.0, self.mass, self.mass, ws[1])
        self.compare(cu, q, out, lse, window, n_first)

    def compare(self, cu, q, out, lse, window, n_first):
        grp = self.hq // self.hk
        for b in range(len(cu) - 1):
            n, mine = self.k[b].shape[0], slice(cu[b], cu[b + 1])
            m = mine.stop - mine.start
            self.want_mass[b] = torch.cat((self.want_mass[b], torch.zeros((self.hk, n - self.want_mass[b].shape[1]), dtype=torch.float64, device="cuda")), 1)
            p, i = torch.arange(n - m, n, device="cuda")[:, None], torch.arange(n, device="cuda")
            ok = i <= p
            if window:
                ok &= (i > p - window) | (i < n_first)
            for h in range(self.hq):
                s = torch.where(ok, self.scale * (q[mine, h].double() @ self.k[b][:, h // grp].double().T.contiguous()), -torch.inf)
                w = torch.softmax(s, 1)
                v = self.v[b][:, h // grp].double()
                mag = w @ v.abs()
                tol = R.STEP[self.dtype] * (w @ v).abs() + mag * (2 * 2.0 ** -8 if self.dtype is BF16 else 2.0 ** -17)      # (as in paged_ref, scores of a few units)
                assert ((out[mine, h].double() - w @ v).abs() <= tol + mag * 1e-5).all()
                assert ((lse[mine, h].double() - torch.logsumexp(s, 1)).abs() <= 1e-5).all()
                self.want_mass[b][h // grp] += w.sum(0)
            got = self.mass[b, :, :n].double()
            assert ((got - self.want_mass[b]).abs() <= 1e-4 * self.want_mass[b] + 1e-6).all()
            assert (self.mass[b, :, n:] == 0).all()

    def evict(self, keep, n_first, n_recent):
        batch, most = len(keep), max(keep)
        lens = [k.shape[0] for k in self.k]
        new_table = torch.full((batch, -(-most // self.page)), -1, dtype=torch.int32, device="cuda")
        for b, n in enumerate(lens):
            for i in range(-(-min(n, keep[b]) // self.page)):
                new_table[b, i] = self.free.pop(0)
        kept, new_len = torch.full((batch, most), -1, dtype=torch.int32, device="cuda"), torch.zeros((batch,), dtype=torch.int32, device="cuda")
        new_mass = torch.zeros((batch, self.hk, most), device="cuda")
        ws = torch.empty((B.kvs_workspace_size("evict_paged", self.shape, batch, self.pages.max_ctx),), dtype=torch.uint8, device="cuda")
        B.kvs_evict_paged(self.shape, self.cache, self.pages, torch.tensor(keep, dtype=torch.int32, device="cuda"), n_first, n_recent, self.mass, new_table, kept, new_len, new_mass, ws)
        old = self.mass.clone()
        self.table.fill_(-1)
        self.mass.zero_()
        for b, n in enumerate(lens):
            rows = R.kept_rows(old[b].cpu(), n, keep[b], n_first, n_recent)
            m = len(rows)
            assert int(new_len[b]) == m and kept[b, :m].tolist() == rows
            at = torch.tensor(rows, device="cuda", dtype=torch.long)
            self.k[b], self.v[b], self.want_mass[b] = self.k[b][at], self.v[b][at], self.want_mass[b][:, at]
            assert torch.equal(new_mass[b, :, :m], old[b][:, at])
            self.mass[b, :, :m] = new_mass[b, :, :m]
            self.table[b, :-(-m // self.page)] = new_table[b, :-(-m // self.page)]
        self.ctx_len.copy_(new_len)


@pytest.mark.parametrize("hq,hk,d,dtype,page", [(8, 2, 128, BF16, 16), (28, 4, 128, BF16, 32), (4, 4, 64, F32, 16), (6, 3, 64, BF16, 64)])
def test_prompts_steps_and_evictions(hq, hk, d, dtype, page):
    loop = Loop(hq, hk, d, dtype, page, 3, 640 // page, 4 * 640 // page)
    loop.step([200, 1, 37])
    loop.step([130, 64, 0])
    loop.step([1, 1, 1])
    loop.evict([120, 50, 60], 4, 20)
    for _ in range(3):
        loop.step([1, 1, 1])
    loop.step([5, 90, 1])
    loop.evict([64, 64, 64], 1, 64)
    loop.step([1, 1, 1], 0, 0)


def test_a_window_over_a_growing_context():
    loop = Loop(8, 2, 128, BF16, 16, 2, 40, 90, seed=3)
    for new in ([150, 30], [100, 1], [1, 1], [1, 1], [64, 200]):
        loop.step(new, 48, 4)


def test_requests_that_share_pages():
    """Two requests over one prefix: its rows are read through both, and an eviction of one leaves the other's as they are."""
    loop = Loop(8, 2, 128, BF16, 16, 2, 20, 60, seed=5)
    loop.step([64, 0])
    loop.table[1, :4] = loop.table[0, :4]
    loop.ctx_len[1] = 64
    loop.k[1], loop.v[1], loop.want_mass[1] = loop.k[0].clone(), loop.v[0].clone(), torch.zeros_like(loop.want_mass[0])
    loop.step([10, 30])
    loop.step([1, 1])
    loop.evict([40, 300], 4, 8)
    loop.step([1, 1])


def test_a_captured_step_and_two_graphs_with_one_workspace():
    """Store, attention and mass of a decode step in one graph; another graph of another layer's calls uses the same workspace."""
    layers = [Loop(8, 2, 128, BF16, 16, 2, 160, 330, seed=s) for s in (7, 8)]
    bufs = []
    ws = None
    for loop in layers:
        loop.step([1500, 700])
        k, v, q = loop.rand(2, 2, 128), loop.rand(2, 2, 128), loop.rand(2, 8, 128)
        out, lse = torch.empty_like(q), torch.empty((2, 8), device="cuda")
        if ws is None:
            ws = torch.empty((B.kvs_workspace_size("attention_paged", loop.shape, 2, loop.pages.max_ctx, 2),), dtype=torch.uint8, device="cuda")

        def call(loop=loop, k=k, v=v, q=q, out=out, lse=lse):
            B.kvs_store_paged(loop.shape, loop.cache, loop.pages, None, None, k, v, loop.mass)
            B.kvs_attention_paged(loop.shape, loop.cache, loop.pages, None, None, q, loop.scale, 0, 0, out, lse, ws)
            B.kvs_mass_paged(loop.shape, loop.cache, loop.pages, None, None, q, lse, loop.scale, 0, 0, 1.0, loop.mass, loop.mass)
        spare = [x.clone() for x in (loop.mass, loop.cache.k, loop.cache.v)]
        call()                                                          # (to load the kernels; undone)
        for x, y in zip((loop.mass, loop.cache.k, loop.cache.v), spare):
            x.copy_(y)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            call()
        bufs.append((loop, k, v, q, out, lse, graph))
    for _ in range(4):
        for loop, k, v, q, *_ in bufs:
            for x in (k, v, q):
                x.copy_(loop.rand(*x.shape))
            for b in range(2):
                loop.grow(b, loop.k[b].shape[0] + 1)
                loop.k[b], loop.v[b] = torch.cat((loop.k[b], k[b:b + 1])), torch.cat((loop.v[b], v[b:b + 1]))
        for *_, graph in bufs:
            graph.replay()
        torch.cuda.synchronize()
        for loop, k, v, q, out, lse, _ in bufs:
            loop.compare([0, 1, 2], q, out, lse, 0, 0)


def test_streams_side_by_side():
    """Two layers on two streams, each with a workspace of its own, and a tensor made on one of them."""
    loops = [Loop(8, 2, 128, BF16, 16, 2, 160, 330, seed=s) for s in (9, 10)]
    for loop in loops:
        loop.step([1500, 700])
    streams = [torch.cuda.Stream() for _ in loops]
    got = []
    for loop, stream in zip(loops, streams):
        k, v, q = loop.rand(300, 2, 128), loop.rand(300, 2, 128), loop.rand(300, 8, 128)
        for b, (lo, hi) in enumerate(((0, 299), (299, 300))):
            loop.grow(b, loop.k[b].shape[0] + hi - lo)
            loop.k[b], loop.v[b] = torch.cat((loop.k[b], k[lo:hi])), torch.cat((loop.v[b], v[lo:hi]))
        cu = torch.tensor([0, 299, 300], dtype=torch.int32, device="cuda")
        out, lse = torch.empty_like(q), torch.empty((300, 8), device="cuda")
        stream.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(stream):
            ws = torch.empty((B.kvs_workspace_size("attention_paged", loop.shape, 2, loop.pages.max_ctx, 300),), dtype=torch.uint8, device="cuda")
            B.kvs_store_paged(loop.shape, loop.cache, loop.pages, cu, None, k, v, loop.mass)
            B.kvs_attention_paged(loop.shape, loop.cache, loop.pages, cu, None, q, loop.scale, 0, 0, out, lse, ws)
            B.kvs_mass_paged(loop.shape, loop.cache, loop.pages, cu, None, q, lse, loop.scale, 0, 0, 1.0, loop.mass, loop.mass, None)
        got.append((q, out, lse))
    torch.cuda.synchronize()
    for loop, (q, out, lse) in zip(loops, got):
        loop.compare([0, 299, 300], q, out, lse, 0, 0)


def test_what_the_binding_refuses():
    c = R.Case(4, 2, 64, BF16, 16, [(40, 1), (20, 1)], seed=1)
    cache, pages = c.on()
    out, lse = torch.empty_like(c.q), torch.empty((2, 4), device="cuda")
    call = lambda **kw: B.kvs_attention_paged(**{**dict(shape=c.shape, cache=cache, pages=pages, cu_new=None, sel_pos=None, q_new=c.q, scale=1.0, window=0, n_first=0, out=out, lse_out=lse), **kw})
    call()
    for kw in (dict(q_new=c.q.float()), dict(q_new=c.q.cpu()), dict(out=out[:1]), dict(out=out.float()), dict(lse_out=lse[:1]), dict(lse_out=lse.double()), dict(sel_pos=c.sel_pos.long()),
               dict(sel_pos=c.sel_pos[:1]), dict(cu_new=torch.zeros((2,), dtype=torch.int32, device="cuda")), dict(q_new=c.q.transpose(0, 1)), dict(out=torch.empty((2, 64, 4), dtype=BF16, device="cuda").transpose(1, 2)),
               dict(shape=B.make_shape(4, 2, 64, B.F32)), dict(shape=B.make_shape(4, 4, 64, B.BF16)), dict(shape=B.make_shape(4, 2, 128, B.BF16))):
        with pytest.raises((TypeError, ValueError)):
            call(**kw)
    for kw in (dict(window=-1), dict(n_first=-2), dict(scale=float("nan")), dict(workspace=torch.empty((600,), dtype=torch.uint8, device="cuda")[16:])):
        with pytest.raises(B.KvsError):
            call(**kw)
    mass = torch.zeros((2, 2, 40), device="cuda")
    for bad in (mass[:, :, :39].contiguous(), mass[:1], mass.double(), torch.zeros((2, 40, 2), device="cuda").transpose(1, 2)):
        with pytest.raises((TypeError, ValueError, B.KvsError)):
            B.kvs_mass_paged(c.shape, cache, pages, None, None, c.q, lse, 1.0, 0, 0, 1.0, None, bad)
    with pytest.raises(ValueError):
        B.kvs_mass_paged(c.shape, cache, pages, None, None, c.q, lse, 1.0, 0, 0, 1.0, torch.zeros((2, 2, 41), device="cuda"), mass)
    with pytest.raises((TypeError, ValueError)):
        B.kvs_store_paged(c.shape, cache, pages, None, None, c.q[:, :2].contiguous(), c.q[:1, :2].contiguous())
    with pytest.raises(ValueError):
        B.kvs_evict_paged(c.shape, cache, pages, torch.zeros((2,), dtype=torch.int32, device="cuda"), 0, 0, mass, torch.zeros((1, 3), dtype=torch.int32, device="cuda"))
    torch.cuda.synchronize()
