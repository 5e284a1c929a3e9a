"""kvs_rotary, kvs_store_kv8, kvs_deviation_kv8, kvs_select_topk and kvs_attention_kv8 as a program uses them together: reused keys
move to where the prompt has them and are stored, fresh rows score them, the best are recomputed, stored and attend, and a few
decode steps append a row each.  Then what the calls promise beside that: other streams, two of them at once, a captured run,
caches and tensors behind 2^32 bytes."""
import numpy as np
import pytest
import torch

import kv8_ref as R
from paper_2503_16525_amd import binding as B
from test_gpu_rotary import _check as check_turned
from test_gpu_rotary import _frequencies

pytestmark = pytest.mark.gpu

CASES = [(8, 2, 128, "bf16", "e4m3", 32), (4, 4, 64, "f32", "int8", 16), (28, 4, 128, "bf16", "int8", 64), (6, 3, 64, "f32", "e4m3", 128)]


class Run:
    """Two requests in one cache; rows behind each for what a decode appends."""

    def __init__(self, hq, hk, d, dtype, code, block, lens=(400, 301), room=8, seed=0):
        self.hq, self.hk, self.d, self.dtype, self.code, self.block, self.lens = hq, hk, d, dtype, code, block, list(lens)
        self.dt = torch.bfloat16 if dtype == "bf16" else torch.float32
        self.shape = B.make_shape(hq, hk, d, B.BF16 if dtype == "bf16" else B.F32)
        self.spec = B.rotary_spec(d, "half", "linear", 10000.0, 2.0)
        self.off = [3, 3 + lens[0] + room]
        self.n_rows = self.off[1] + lens[1] + room
        self.n, self.take = sum(lens), [x // 8 for x in lens]
        self.gen = torch.Generator().manual_seed(seed)
        at = [torch.arange(o, o + x) for o, x in zip(self.off, lens)]
        self.rows = torch.cat(at).to(torch.int32).cuda()                 # the prompts' cache rows
        self.pos = torch.cat([torch.arange(x) for x in lens]).to(torch.int32).cuda()
        self.old = torch.randint(0, 5000, (self.n,), generator=self.gen, dtype=torch.int32).cuda()
        self.k_old, self.v_old, self.k_fresh, self.v_fresh = (self.randn(self.n, hk) for _ in range(4))
        self.v_fresh = (self.v_old.float() + 0.2 * self.v_fresh.float() * self.randn(self.n, 1).float().exp()).to(self.dt)
        self.q = (self.randn(self.n, hq).float() / d ** 0.5).to(self.dt)
        self.cache = B.Cache8.empty(self.shape, self.n_rows, block, B.E4M3 if code == "e4m3" else B.INT8)
        self.k_moved = torch.empty_like(self.k_old)
        self.reused = torch.ones((self.n_rows,), dtype=torch.uint8).cuda()
        self.dev_v, self.score = torch.empty((hk, lens[0])).cuda(), torch.full((self.n,), -torch.inf).cuda()
        self.idx = torch.empty((sum(self.take),), dtype=torch.int32).cuda()
        n_sel = sum(self.take)
        self.q_out, self.k_out = torch.empty((n_sel, hq, d), dtype=self.dt).cuda(), torch.empty((n_sel, hk, d), dtype=self.dt).cuda()
        self.out, self.lse = torch.empty_like(self.q_out), torch.empty((n_sel, hq)).cuda()
        self.ws = torch.empty((B.kvs_workspace_size("attention_kv8", self.shape, 2, self.n_rows, n_sel),), dtype=torch.uint8, device="cuda")
        self.first = torch.cat([torch.full((t,), o) for t, o in zip(self.take, self.off)]).to(torch.int32).cuda()
        self.entry = torch.cat([torch.full((t,), sum(lens[:b])) for b, t in enumerate(self.take)]).cuda()

    def randn(self, n, heads):
        return torch.randn((n, heads, self.d), generator=self.gen).to(self.dt).cuda()

    def clear(self):
        for x in (self.cache.k.view(torch.uint8), self.cache.v.view(torch.uint8), self.cache.k_scale, self.cache.v_scale):
            x.zero_()
        self.reused.fill_(1)

    def reuse(self):
        B.kvs_rotary(self.shape, self.spec, self.pos, self.old, None, self.k_old, None, self.k_moved)
        B.kvs_store_kv8(self.shape, self.cache, self.k_moved, self.v_old, self.rows)

    def choose(self):
        at = 0
        for o, x in zip(self.off, self.lens):
            B.kvs_deviation_kv8(self.shape, self.cache, o, x, None, self.v_fresh[at:at + x], self.reused[o:o + x], None, B.SCORE_V,
                                None, self.dev_v.view(-1)[:self.hk * x].view(self.hk, x), self.score[at:at + x])
            at += x
        B.kvs_select_topk(self.score, [0, self.lens[0], self.n], self.take, self.idx)

    def recompute(self):
        s = self.entry + self.idx
        self.k_sel, self.v_sel, self.q_sel = self.k_fresh[s], self.v_fresh[s], self.q[s]
        B.kvs_rotary(self.shape, self.spec, self.idx, None, self.q_sel, self.k_sel, self.q_out, self.k_out)
        B.kvs_store_kv8(self.shape, self.cache, self.k_out, self.v_sel, self.first + self.idx, 0, self.reused)
        B.kvs_attention_kv8(self.shape, self.cache, self.off, self.lens, [0, self.take[0], sum(self.take)], self.q_out, self.idx, 1.0, self.out, self.lse, self.ws)

    def all(self):
        self.reuse()
        self.choose()
        self.recompute()

    def state(self):
        c = self.cache
        return [x.clone() for x in (c.k.view(torch.uint8), c.v.view(torch.uint8), c.k_scale, c.v_scale, self.reused, self.idx, self.out, self.lse)]


def _n(x):
    return x.float().cpu().numpy()


@pytest.mark.parametrize("hq,hk,d,dtype,code,block", CASES)
def test_a_request_as_it_runs(hq, hk, d, dtype, code, block):
    r = Run(hq, hk, d, dtype, code, block)
    kc, vc = (np.zeros((r.n_rows, hk, d), np.uint8) for _ in range(2))
    ks, vs = (np.zeros((-(-r.n_rows // block), hk), np.float32) for _ in range(2))

    def stored(k, v, at, what):
        R.store(kc, ks, _n(k), at, block, code)
        R.store(vc, vs, _n(v), at, block, code)
        for got, want in ((r.cache.k.view(torch.uint8), kc), (r.cache.k_scale, ks), (r.cache.v.view(torch.uint8), vc), (r.cache.v_scale, vs)):
            np.testing.assert_array_equal(got.cpu().numpy(), want, err_msg=what)

    def attended(q, pos, lens, cu, out, lse, what):
        kh, vh = R.held(kc, ks, block, code), R.held(vc, vs, block, code)
        q = q.double().cpu().numpy()
        ref = R.joined([R.attention(q[cu[b]:cu[b + 1]], pos[cu[b]:cu[b + 1]], kh[o:o + x], vh[o:o + x], 1.0) for b, (o, x) in enumerate(zip(r.off, lens))])
        R.check_attention(_n(out), _n(lse), ref, dtype, max(lens), what)

    f = _frequencies(d, "linear", 10000.0, 2.0)
    r.reuse()
    check_turned(r.k_moved, r.k_old, (r.pos - r.old).double().cpu().numpy(), f, "half", 1.0, "the move")
    stored(r.k_moved, r.v_old, r.rows.tolist(), "the reused rows")
    r.choose()
    # 2^-24 times 14 roundings and one for each head, as in the deviation's own test
    want = np.abs(_n(r.v_fresh).astype(np.float64) - R.held(vc, vs, block, code)[r.rows.cpu().numpy()]).sum((1, 2))
    np.testing.assert_allclose(_n(r.score), want, rtol=(16 + hk) * 2.0 ** -24)
    score, idx, at = _n(r.score), r.idx.cpu().numpy(), 0
    for b, x in enumerate(r.lens):
        mine = score[sum(r.lens[:b]):][:x]
        np.testing.assert_array_equal(idx[at:at + r.take[b]], np.sort(np.argsort(-mine, kind="stable")[:r.take[b]]))
        at += r.take[b]
    r.recompute()
    check_turned(r.q_out, r.q_sel, idx.astype(np.float64), f, "half", 1.0, "Q")
    check_turned(r.k_out, r.k_sel, idx.astype(np.float64), f, "half", 1.0, "K")
    chosen = (r.first.cpu().numpy() + idx).tolist()
    stored(r.k_out, r.v_sel, chosen, "the recomputed rows")
    left = np.ones(r.n_rows, np.uint8)
    left[chosen] = 0
    np.testing.assert_array_equal(r.reused.cpu().numpy(), left)
    attended(r.q_out, idx, r.lens, [0, r.take[0], sum(r.take)], r.out, r.lse, "the recomputed rows")
    lens = list(r.lens)
    for step in range(4):                                  # the second request has ended behind the second step: its place stays in the batch
        live = [True, step < 2]
        rows = torch.tensor([o + x if on else -1 for o, x, on in zip(r.off, lens, live)], dtype=torch.int32).cuda()
        pos = torch.tensor([x if on else -1 for x, on in zip(lens, live)], dtype=torch.int32).cuda()
        q, k, v = (r.randn(2, hq).float() / d ** 0.5).to(r.dt), r.randn(2, hk), r.randn(2, hk)
        qo, ko, out, lse = torch.empty_like(q), torch.empty_like(k), torch.full_like(q, 7.0), torch.full((2, hq), 7.0).cuda()
        B.kvs_rotary(r.shape, r.spec, pos, None, q, k, qo, ko)
        B.kvs_store_kv8(r.shape, r.cache, ko, v, rows)
        stored(ko, v, rows.tolist(), f"step {step}")
        lens = [x + on for x, on in zip(lens, live)]
        B.kvs_attention_kv8(r.shape, r.cache, r.off, lens, [0, 1, 2], qo, pos, 1.0, out, lse, r.ws)
        attended(qo, pos.tolist(), lens, [0, 1, 2], out, lse, f"step {step}")
        if not live[1]:
            assert not out[1].any() and torch.isneginf(lse[1]).all()


@pytest.mark.parametrize("hq,hk,d,dtype,code,block", CASES[:2])
def test_the_run_captured_and_replayed(hq, hk, d, dtype, code, block):
    r = Run(hq, hk, d, dtype, code, block)
    r.clear()
    r.all()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        r.all()
    for i in range(3):
        r.q.mul_(-1.1)
        r.v_fresh.copy_(torch.roll(r.v_fresh, 7, 0))
        r.clear()
        r.all()
        want = r.state()
        r.clear()
        r.out.fill_(7.0)
        g.replay()
        torch.cuda.synchronize()
        for a, b in zip(r.state(), want):
            assert torch.equal(a, b), i


def test_two_streams_at_once():
    """Two runs, each on a stream of its own that is not the current one's, enqueued side by side."""
    runs = [Run(*CASES[i % 2], lens=(900, 777), seed=i) for i in range(4)]
    want = []
    for r in runs:
        r.clear()
        r.all()
        want.append(r.state())
        r.clear()
        r.out.fill_(7.0)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for step in ("reuse", "choose", "recompute"):
        for i, r in enumerate(runs):
            with torch.cuda.stream(streams[i % 2]):
                getattr(r, step)()
    torch.cuda.synchronize()
    for r, w in zip(runs, want):
        for a, b in zip(r.state(), w):
            assert torch.equal(a, b)


def test_a_stream_given_by_its_handle():
    r = Run(*CASES[0])
    r.clear()
    r.all()
    want = r.state()
    s = torch.cuda.Stream()
    r.out.fill_(7.0)
    torch.cuda.synchronize()
    B.kvs_attention_kv8(r.shape, r.cache, r.off, r.lens, [0, r.take[0], sum(r.take)], r.q_out, r.idx, 1.0, r.out, r.lse, r.ws, stream=s.cuda_stream)
    s.synchronize()
    assert torch.equal(r.out, want[6]) and torch.equal(r.lse, want[7])


@pytest.mark.parametrize("code", ["e4m3", "int8"])
def test_caches_behind_32_bits(code):
    """The last rows of a cache of 4.6 GB a tensor answer as the same rows of a small one."""
    hq, hk, d, block, n = 32, 8, 128, 32, 2048
    big, small = 4_500_000 // block * block, n
    sh, kind = B.make_shape(hq, hk, d, B.BF16), B.E4M3 if code == "e4m3" else B.INT8
    gen = torch.Generator().manual_seed(2)
    k, v = (torch.randn((n, hk, d), generator=gen).to(torch.bfloat16).cuda() for _ in range(2))
    q = (torch.randn((64, hq, d), generator=gen) / d ** 0.5).to(torch.bfloat16).cuda()
    pos = torch.randperm(n, generator=gen)[:64].sort().values.to(torch.int32).cuda()
    some = torch.arange(0, n, 5, dtype=torch.int32).cuda()
    got = []
    for rows in (small, big):
        c, at = B.Cache8.empty(sh, rows, block, kind), rows - n
        assert rows == small or c.k.numel() > 1 << 32
        B.kvs_store_kv8(sh, c, k, v, None, at)
        B.kvs_store_kv8(sh, c, v[:some.numel()], k[:some.numel()], some + at)
        dev, score = torch.empty((hk, n)).cuda(), torch.empty((n,)).cuda()
        B.kvs_deviation_kv8(sh, c, at, n, None, v, None, None, B.SCORE_V, None, dev, score)
        one, all64 = torch.empty((1, hq, d), dtype=torch.bfloat16).cuda(), torch.empty_like(q)
        lse = torch.empty((64, hq)).cuda()
        ws = torch.empty((B.kvs_workspace_size("attention_kv8", sh, 1, rows, 64),), dtype=torch.uint8, device="cuda")
        B.kvs_attention_kv8(sh, c, [at], [n], [0, 1], q, pos[63:], 1.0, one, None, ws)
        B.kvs_attention_kv8(sh, c, [at], [n], [0, 64], q, pos, 1.0, all64, lse, ws)
        torch.cuda.synchronize()
        got.append([c.k[at:].view(torch.uint8).clone(), c.v[at:].view(torch.uint8).clone(), c.k_scale[at // block:].clone(), dev, score, one, all64, lse])
        del c
    for a, b in zip(*got):
        assert torch.equal(a, b)


def test_rotary_behind_32_bits():
    """600000 rows of 32 heads: 4.9 GB."""
    n, hq, hk, d = 600_000, 32, 1, 128
    sh, spec = B.make_shape(hq, hk, d, B.BF16), B.rotary_spec(d)
    q = torch.empty((n, hq, d), dtype=torch.bfloat16, device="cuda").normal_()
    pos = torch.arange(n, dtype=torch.int32).cuda()
    out = torch.empty_like(q)
    B.kvs_rotary(sh, spec, pos, None, q, None, out, None)
    for at in (0, 262_140, 524_280, n - 50):               # the second and third lie around 2^30 and 2^31 elements
        want = torch.empty((50, hq, d), dtype=torch.bfloat16, device="cuda")
        B.kvs_rotary(sh, spec, pos[at:at + 50], None, q[at:at + 50], None, want, None)
        torch.cuda.synchronize()
        assert torch.equal(out[at:at + 50], want), at


def test_rotary_of_more_pairs_than_a_launch_has_threads():
    """A turned part of 100 channels goes by single pairs: 900000 rows of 64 heads are 4.5e9 of them and of the channels passed through."""
    n, hq, d = 900_000, 64, 128
    sh, spec = B.make_shape(hq, hq, d, B.BF16), B.rotary_spec(100)
    q = torch.empty((n, hq, d), dtype=torch.bfloat16, device="cuda").normal_()
    pos, old = torch.arange(n, dtype=torch.int32).cuda(), (torch.arange(n, dtype=torch.int32) % 1013).cuda()
    out = torch.full_like(q, 7.0)
    B.kvs_rotary(sh, spec, pos, old, q, None, out, None)
    for at in (0, 430_000, 860_320, n - 50):               # a launch has 860370 of them
        want = torch.empty((50 if at != 860_320 else 100, hq, d), dtype=torch.bfloat16, device="cuda")
        part = slice(at, at + want.shape[0])
        B.kvs_rotary(sh, spec, pos[part], old[part], q[part], None, want, None)
        torch.cuda.synchronize()
        assert torch.equal(out[part], want), at
