"""What the rotary and 8-bit-cache calls refuse, on the host, before anything is enqueued (no GPU: every call below fails its
checks or has nothing to do)."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2503_16525_amd import binding as B

FAKE = 0x10000


@pytest.fixture(scope="module")
def lib():
    return B.load()


def _shape(hq=32, hk=8, d=128, dt=B.BF16):
    return B.make_shape(hq, hk, d, dt)


def _cache(k=FAKE, v=FAKE, ks=FAKE, vs=FAKE, n=1000, block=32, code=0):
    return B._Cache8(k, v, ks, vs, n, block, code)


def test_rotary_refusals(lib):
    def call(shape=_shape(), spec=None, n=10, pos=FAKE, q=FAKE, qs=4096, k=FAKE * 16, ks=1024, qo=FAKE * 64, qos=4096, ko=FAKE * 128, kos=1024, **kw):
        spec = spec if spec is not None else B.rotary_spec(**{**dict(rotary_dim=128), **kw})
        return lib.kvs_rotary(ctypes.byref(shape), ctypes.byref(spec), n, pos, None, q, qs, k, ks, qo, qos, ko, kos, None)
    assert call(n=0, pos=None, q=None, k=None) == B.OK
    assert call(n=-1) == B.EINVAL
    assert call(pos=None) == B.EINVAL
    assert call(q=None, k=None) == B.EINVAL and b"neither" in lib.kvs_last_error()
    assert call(qo=None) == B.EINVAL
    assert call(q=FAKE + 2) == B.EINVAL
    assert call(shape=_shape(d=96)) == B.EUNSUPPORTED
    for r in (0, 3, 130, -2):
        assert call(rotary_dim=r) == B.EINVAL, r
    assert call(qs=4095) == B.EINVAL                       # shorter than a row
    assert call(qs=4100) == B.EINVAL                       # rows that begin between 16-byte pieces
    assert call(kos=512) == B.EINVAL
    assert call(qs=1 << 45) == B.EINVAL                    # the tensor would leave the address space
    assert call(qo=FAKE + 4096) == B.EINVAL and b"overlaps" in lib.kvs_last_error()
    assert call(qo=FAKE, qos=8192) == B.EINVAL             # the same pointer, another stride
    for kw in (dict(base=1.0), dict(base=float("nan")), dict(base=float("inf")), dict(magnitude=float("inf")), dict(magnitude=1e300),
               dict(scaling="linear", factor=0.0), dict(scaling="ntk", factor=2.0, rotary_dim=2), dict(scaling="ramp", original=0),
               dict(scaling="ramp", original=100, low=0.0), dict(scaling="wavelength", original=100, low=4.0, high=4.0),
               dict(scaling="wavelength", original=100, low=1.0, high=float("inf"))):
        assert call(**kw) == B.EINVAL, kw
    bad = B.rotary_spec(128)
    bad.layout = 2
    assert call(spec=bad) == B.EINVAL
    bad = B.rotary_spec(128)
    bad.scaling = 5
    assert call(spec=bad) == B.EINVAL
    assert lib.kvs_rotary(ctypes.byref(_shape()), None, 1, FAKE, None, FAKE, 4096, None, 0, FAKE * 64, 4096, None, 0, None) == B.EINVAL


CALLS = ["store", "deviation", "attention"]


@pytest.mark.parametrize("call", CALLS)
def test_cache_refusals(lib, call):
    one = np.array([0], np.int64)
    ln, cu = np.array([10], np.int64), np.array([0, 1], np.int64)

    def with_cache(c, shape=_shape()):
        c = ctypes.byref(c) if c is not None else None
        sh = ctypes.byref(shape)
        if call == "store":
            return lib.kvs_store_kv8(sh, c, None, FAKE, None, 0, 10, None, None, None)
        if call == "deviation":
            return lib.kvs_deviation_kv8(sh, c, 0, 10, None, None, None, None, 0, None, FAKE, None, None)
        return lib.kvs_attention_kv8(sh, c, 1, one.ctypes.data, ln.ctypes.data, cu.ctypes.data, None, FAKE, 1.0, FAKE, None, None, 0, None)
    assert with_cache(None) == B.EINVAL
    for kw, word in ((dict(code=2), b"code"), (dict(block=8), b"block"), (dict(block=48), b"block"), (dict(block=256), b"block"), (dict(n=-1), b"n_rows"),
                     (dict(k=None), b"NULL"), (dict(vs=None), b"NULL"), (dict(v=FAKE + 8), b"aligned"), (dict(ks=FAKE + 2), b"scales")):
        assert with_cache(_cache(**kw)) == B.EINVAL and word in lib.kvs_last_error(), kw
    assert with_cache(_cache(n=1 << 50)) == B.EUNSUPPORTED
    assert with_cache(_cache(), _shape(hq=65, hk=65)) == B.EUNSUPPORTED
    assert with_cache(_cache(), _shape(dt=5)) == B.EINVAL
    assert with_cache(_cache()) == B.EINVAL and b"NULL" in lib.kvs_last_error()       # the call's own tensors


def test_store_refusals(lib):
    def call(n=10, row0=0, pos=None, k=FAKE, v=FAKE, cache=_cache()):
        return lib.kvs_store_kv8(ctypes.byref(_shape()), ctypes.byref(cache), k, v, pos, row0, n, None, None, None)
    assert call(n=0, k=None) == B.OK
    assert call(n=-1) == B.EINVAL
    assert call(n=1 << 31, pos=FAKE) == B.EINVAL
    assert call(row0=-1) == B.EINVAL
    assert call(row0=991) == B.EINVAL
    assert call(n=1001) == B.EINVAL
    assert call(k=None) == B.EINVAL
    assert call(v=FAKE + 8) == B.EINVAL
    assert call(cache=_cache(k=None, v=None, ks=None, vs=None, n=0), n=0) == B.OK
    # every entry of a list lies outside an empty cache
    assert call(cache=_cache(k=None, v=None, ks=None, vs=None, n=0), n=5, pos=FAKE, k=None) == B.OK


def test_deviation_refusals(lib):
    def call(n=10, row0=0, mode=0, kf=None, vf=FAKE, dk=None):
        return lib.kvs_deviation_kv8(ctypes.byref(_shape()), ctypes.byref(_cache()), row0, n, kf, vf, None, None, mode, dk, FAKE, FAKE, None)
    assert call(n=0, vf=None) == B.OK
    assert call(n=-1) == B.EINVAL
    assert call(row0=-1) == B.EINVAL
    assert call(row0=995) == B.EINVAL
    assert call(mode=2) == B.EINVAL
    assert call(vf=None) == B.EINVAL
    assert call(mode=1) == B.EINVAL and b"k_fresh" in lib.kvs_last_error()
    assert call(dk=FAKE) == B.EINVAL
    assert call(mode=1, kf=FAKE + 4) == B.EINVAL
    assert call(vf=FAKE + 4) == B.EINVAL


def test_attention_refusals(lib):
    def call(off=(0,), ln=(100,), cu=(0, 5), q=FAKE, pos=FAKE, scale=1.0, out=FAKE, ws=None, ws_bytes=0, batch=None, cache=_cache(), shape=_shape()):
        o, n, c = (np.array(x, np.int64) for x in (off, ln, cu))
        return lib.kvs_attention_kv8(ctypes.byref(shape), ctypes.byref(cache), len(off) if batch is None else batch, o.ctypes.data, n.ctypes.data, c.ctypes.data,
                                     q, pos, scale, out, None, ws, ws_bytes, None)
    assert call(batch=0) == B.OK
    assert call(batch=-1) == B.EINVAL
    assert call(cu=(0, 0), q=None, pos=None, out=None) == B.OK
    assert call(cu=(1, 5)) == B.EINVAL
    assert call(off=(0, 0), ln=(10, 10), cu=(0, 5, 3)) == B.EINVAL
    assert call(off=(-1,)) == B.EINVAL
    assert call(ln=(-1,)) == B.EINVAL
    assert call(off=(901,)) == B.EINVAL and b"outside" in lib.kvs_last_error()
    assert call(cache=_cache(n=1 << 28), ln=((1 << 31),)) == B.EINVAL
    assert call(cu=(0, 1 << 27)) == B.EINVAL               # 2^27 tokens of 32 heads: rows past 32 bits
    for s in (float("nan"), float("inf")):
        assert call(scale=s) == B.EINVAL
    for kw in (dict(q=None), dict(pos=None), dict(out=None), dict(q=FAKE + 4), dict(out=FAKE + 8), dict(ws=FAKE * 16 + 64, ws_bytes=1 << 20)):
        assert call(**kw) == B.EINVAL, kw


def test_the_workspace_never_shrinks_with_the_totals():
    for sh in (_shape(), _shape(hq=28, hk=4), _shape(hq=4, hk=4, d=64, dt=B.F32)):
        for n_sel in (1, 64, 5000):
            sizes = [B.kvs_workspace_size("attention_kv8", sh, 1, n, n_sel) for n in (0, 1, 31, 32, 1000, 4096, 131072, 1 << 21)]
            assert sizes == sorted(sizes)
            if n_sel == 1 or sh.dtype == B.F32:            # pieces only; from 7373 rows on there is room for a bf16 copy
                assert sizes[-1] <= 2048 * 32 * (4 * sh.head_dim + 16)
            elif n_sel == 5000:
                assert sizes[-1] >= 512 * sh.n_kv_heads << 21
        for n in (1, 4096, 131072):
            sizes = [B.kvs_workspace_size("attention_kv8", sh, 1, n, n_sel) for n_sel in (0, 1, 2, 63, 64, 5000, 1 << 20, 1 << 40)]
            assert sizes == sorted(sizes)
    assert B.kvs_workspace_size("attention_kv8", None, 1, 10, 10) == 0


def test_binding_refusals():
    f8, i8 = torch.zeros((40, 8, 128), dtype=torch.uint8).view(torch.float8_e4m3fn), torch.zeros((40, 8, 128), dtype=torch.int8)
    s = torch.zeros((3, 8))
    for args, err in (((f8, i8, s, s, 16), TypeError), ((f8.view(torch.uint8), f8.view(torch.uint8), s, s, 16), TypeError), ((f8, f8[:39], s, s, 16), ValueError),
                      ((i8, i8, s[:2], s, 16), ValueError), ((i8, i8, s, s, 32), ValueError), ((i8, i8, s, s, 0), ValueError)):
        with pytest.raises(err):
            B.Cache8(*args)
    with pytest.raises(KeyError):
        B.rotary_spec(64, layout="other")
