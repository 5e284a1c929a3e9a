"""What the calls on a cache in pages refuse, on the host, before anything is enqueued (no GPU: every call below fails its checks or has
nothing to do)."""
import ctypes

import pytest
import torch

import paged_ref as R
from paper_2503_16525_amd import binding as B

FAKE = 0x10000
CALLS = ["store", "attention", "mass", "evict"]


@pytest.fixture(scope="module")
def lib():
    return B.load()


def _call(lib, name, shape=None, k=FAKE, v=FAKE, n_pages=100, page=16, table=FAKE, ctx_len=FAKE, max_ctx=1000, batch=4, width=80, cu=FAKE, sel=None, n=10, q=FAKE, out=FAKE, scale=0.1,
          window=0, n_first=0, ws=None, ws_bytes=0, mass=FAKE, stride=1000, decay=1.0, lse=FAKE, mass_out=FAKE, keep=FAKE, max_keep=500, recent=0, new_table=None, new_width=0,
          cache=True, pages=True, new_mass=None):
    shape = shape or B.make_shape(32, 8, 128, B.BF16)
    s = ctypes.byref(shape)
    c = ctypes.byref(B._PagedCache(k, v, n_pages, page)) if cache else None
    p = ctypes.byref(B._PageTable(table, ctx_len, max_ctx, batch, width)) if pages else None
    if name == "store":
        return lib.kvs_store_paged(s, c, p, cu, sel, n, q, q, mass, stride, None)
    if name == "attention":
        return lib.kvs_attention_paged(s, c, p, cu, sel, n, q, scale, window, n_first, out, lse, ws, ws_bytes, None)
    if name == "mass":
        return lib.kvs_mass_paged(s, c, p, cu, sel, n, q, lse, scale, window, n_first, decay, mass, mass_out, stride, ws, ws_bytes, None)
    return lib.kvs_evict_paged(s, c, p, keep, max_keep, n_first, recent, mass, stride, new_table, new_width, None, None, new_mass, ws, ws_bytes, None)


@pytest.mark.parametrize("name", CALLS)
def test_refusals_of_every_call(lib, name):
    call = lambda **kw: _call(lib, name, **kw)
    assert call(batch=0, n=0, cu=None) == B.OK
    assert call(cache=False) == B.EINVAL and call(pages=False) == B.EINVAL
    assert call(shape=B.make_shape(30, 8, 128, B.BF16)) == B.EINVAL
    assert call(shape=B.make_shape(32, 8, 96, B.BF16)) == B.EUNSUPPORTED
    assert call(shape=B.make_shape(65, 65, 64, B.BF16)) == B.EUNSUPPORTED
    assert call(shape=B.make_shape(8192, 8, 64, B.BF16)) == B.EUNSUPPORTED
    assert call(shape=B.make_shape(32, 8, 128, 2)) == B.EINVAL
    for page in (0, -16, 8, 24, 48, 512):
        assert call(page=page) == B.EINVAL, page
    assert call(n_pages=-1) == B.EINVAL
    assert call(n_pages=1 << 31) == B.EINVAL
    assert call(batch=-1) == B.EINVAL and call(width=-1) == B.EINVAL and call(max_ctx=-1) == B.EINVAL
    assert call(max_ctx=1 << 31) == B.EINVAL
    assert call(table=None) == B.EINVAL and call(ctx_len=None) == B.EINVAL
    assert call(k=None) == B.EINVAL and call(v=None) == B.EINVAL
    assert call(k=FAKE + 8) == B.EINVAL
    assert b"kvs_" + name.encode() + b"_paged" in lib.kvs_last_error()


@pytest.mark.parametrize("name", ["store", "attention", "mass"])
def test_refusals_of_tokens(lib, name):
    call = lambda **kw: _call(lib, name, **kw)
    assert call(n=-1) == B.EINVAL
    assert call(cu=None, n=10) == B.EINVAL
    assert call(n=1 << 40) == B.EINVAL
    assert call(q=None) == B.EINVAL
    assert call(q=FAKE + 4) == B.EINVAL
    if name != "mass":
        assert call(n=0) == B.OK
    if name != "store":
        assert call(window=-1) == B.EINVAL and call(n_first=-1) == B.EINVAL
        for scale in (float("nan"), float("inf"), -3e38):
            assert call(scale=scale) == B.EINVAL
        assert call(ws=FAKE + 16, ws_bytes=1000) == B.EINVAL


def test_refusals_of_one_call(lib):
    assert _call(lib, "store", stride=999) == B.EINVAL
    for q, out in ((FAKE, FAKE), (FAKE, FAKE + 10 * 32 * 256 - 16), (FAKE + 16, FAKE)):
        assert _call(lib, "attention", q=q, out=out) == B.EINVAL and b"overlaps" in lib.kvs_last_error()
    assert _call(lib, "attention", out=None) == B.EINVAL and _call(lib, "attention", out=FAKE + 2) == B.EINVAL
    assert _call(lib, "mass", stride=999) == B.EINVAL
    assert _call(lib, "mass", lse=None) == B.EINVAL and _call(lib, "mass", mass_out=None) == B.EINVAL
    for decay in (-0.5, float("nan"), float("inf")):
        assert _call(lib, "mass", decay=decay) == B.EINVAL
    evict = lambda **kw: _call(lib, "evict", **{**dict(ws=FAKE, ws_bytes=1 << 30), **kw})
    assert evict(ws=None, ws_bytes=0) == B.EWORKSPACE and evict(ws_bytes=1000) == B.EWORKSPACE and evict(ws=FAKE + 128) == B.EINVAL
    assert evict(stride=999) == B.EINVAL
    assert evict(max_keep=-1) == B.EINVAL and evict(max_keep=1 << 31) == B.EINVAL
    assert evict(n_first=-1) == B.EINVAL and evict(recent=-1) == B.EINVAL
    assert evict(keep=None) == B.EINVAL and evict(mass=None) == B.EINVAL
    assert evict(new_table=FAKE, new_width=31) == B.EINVAL            # 496 rows for 500
    assert evict(new_mass=FAKE) == B.EINVAL                           # ... in place
    assert evict(batch=70000) == B.EINVAL


def test_refusals_of_outputs_over_inputs(lib):
    q, rows = 0x100000, 10 * 32                              # ten tokens of 32 heads
    attention = lambda **kw: _call(lib, "attention", q=q, **kw)
    assert attention(out=q + rows * 256 - 16, lse=None) == B.EINVAL and b"out overlaps" in lib.kvs_last_error()
    assert attention(out=q + rows * 256, lse=q + rows * 256 - 4) == B.EINVAL and b"lse_out overlaps" in lib.kvs_last_error()
    assert attention(out=q + rows * 256, lse=q + 2 * rows * 256 - 4) == B.EINVAL and b"lse_out overlaps" in lib.kvs_last_error()
    assert _call(lib, "mass", mass=FAKE, mass_out=FAKE + 4) == B.EINVAL and b"mass_out overlaps" in lib.kvs_last_error()
    assert _call(lib, "mass", mass=FAKE + 4 * 8 * 1000 * 4 - 4, mass_out=FAKE) == B.EINVAL and b"mass_out overlaps" in lib.kvs_last_error()
    assert _call(lib, "evict", new_mass=FAKE + 4 * 8 * 1000 * 4 - 4) == B.EINVAL and b"new_mass overlaps" in lib.kvs_last_error()
    assert _call(lib, "evict", mass=FAKE + 4 * 8 * 500 * 4 - 4, new_mass=FAKE) == B.EINVAL and b"new_mass overlaps" in lib.kvs_last_error()
    assert _call(lib, "evict", new_mass=FAKE + 4 * 8 * 1000 * 4) == B.EWORKSPACE         # behind it


def test_workspace_sizes(lib):
    sh = B.make_shape(32, 8, 128, B.BF16)
    for call in ("attention_paged", "mass_paged", "evict_paged"):
        sizes = [B.kvs_workspace_size(call, sh, 4, n, 8) for n in (1, 100, 5000, 100000)]
        assert all(x > 0 and x % 256 == 0 for x in sizes)
        assert sizes == sorted(sizes)
        sizes = [B.kvs_workspace_size(call, sh, 4, 5000, n) for n in (1, 8, 100, 5000, 100000, 3000000)]
        assert sizes == sorted(sizes)
        assert B.kvs_workspace_size(call, None, 4, 100, 8) == 0
    assert B.kvs_workspace_size("evict_paged", sh, 4, 100000) >= 4 * 100000 * 8


def test_the_binding_refuses_what_does_not_fit():
    k = torch.zeros((4, 16, 2, 64))
    with pytest.raises((TypeError, ValueError)):
        B.PagedCache(k.half(), k.half())
    with pytest.raises((TypeError, ValueError)):
        B.PagedCache(k, k[:, :, :, :32])
    with pytest.raises((TypeError, ValueError)):
        B.PagedCache(k, k.bfloat16())
    with pytest.raises(TypeError):
        B.PagedCache(k, k)                                              # not on a device
    with pytest.raises(ValueError):
        B.PageTable(torch.zeros((3, 4), dtype=torch.int32), torch.zeros((2,), dtype=torch.int32), 10)


def test_the_reference_against_brute_force():
    """The tests' own reference, on the CPU: every weight from its definition, with a page of nobody in the middle, and what is kept
    by comparison of every pair."""
    for window, n_first in ((0, 0), (3, 0), (3, 2), (1, 50), (100, 1)):
        c = R.Case(4, 2, 64, torch.float32, 16, [(37, [0, 5, 36, -1, 50]), (0, [0]), (20, 3)], seed=window, device="cpu")
        bad = [torch.zeros((n,), dtype=torch.bool) for n in c.lens]
        bad[0][16:32] = True
        out, lse, mag, _ = R.attention(c, window, n_first, bad)
        m, new, _ = R.mass(c, lse, torch.zeros((3, 2, 37)), 1.0, window, n_first, bad)
        for b, n in enumerate(c.lens):
            k, v = c.rows(b)
            got = torch.zeros((2, n), dtype=torch.float64)
            for t, p in enumerate(c.pos[b]):
                s = c.cu[b] + t
                p = min(p, n - 1)
                see = [i for i in range(n) if i <= p and not bad[b][i] and (window == 0 or p - i < window or i < n_first)]
                for h in range(4):
                    e = [torch.exp(c.scale * (c.q[s, h].double() * k[i, h // 2]).sum()) for i in see]
                    if not see:
                        assert lse[s, h] == -torch.inf and (out[s, h] == 0).all()
                        continue
                    total = sum(e)
                    assert abs(float(lse[s, h] - total.log())) < 1e-12
                    assert (out[s, h] - sum(x * v[i, h // 2] for x, i in zip(e, see)) / total).abs().max() < 1e-12
                    for x, i in zip(e, see):
                        got[h // 2, i] += x / total
            assert (new[b, :, :n] - got).abs().max() < 1e-12 if n else True
    w = torch.tensor([[3.0, 1.0, 1.0, 2.0, 1.0, 9.0, 1.0]])
    assert R.kept_rows(w, 7, 4, 1, 1) == [0, 3, 5, 6]
    assert R.kept_rows(w, 7, 5, 0, 0) == [0, 1, 2, 3, 5]
    assert R.kept_rows(w, 7, 3, 2, 5) == [0, 1, 6] and R.kept_rows(w, 7, -1, 2, 5) == [] and R.kept_rows(w, 7, 99, 2, 5) == list(range(7))
    assert R.kept_rows(torch.tensor([[1.0, float("nan"), -torch.inf, 0.5]]), 4, 3, 0, 0) == [0, 2, 3]
