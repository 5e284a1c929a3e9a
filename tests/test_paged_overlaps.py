"""What the calls on a cache in pages write may lie over nothing that they read: refused on the host, before anything is enqueued (no GPU: every
call below fails its checks)."""
import ctypes

import pytest

from paper_2503_16525_amd import binding as B

MB = 1 << 20
N, BATCH, CTX, PAGES, PAGE, HQ, HK, D = 10, 4, 1000, 100, 16, 32, 8, 128
POOL, Q, NEW, LSE, MASS, TABLE, INTS = PAGES * PAGE * HK * D * 2, N * HQ * D * 2, N * HK * D * 2, N * HQ * 4, BATCH * HK * CTX * 4, BATCH * 80 * 4, BATCH * 4
# name -> address, bytes: 16 MB apart from each other
SIZES = dict(k=POOL, v=POOL, q=Q, out=Q, k_new=NEW, v_new=NEW, lse=LSE, lse_out=LSE, mass=MASS, mass_out=MASS, new_mass=BATCH * HK * 500 * 4, kept=BATCH * 500 * 4, new_len=INTS, keep=INTS,
             table=TABLE, ctx_len=INTS, new_table=BATCH * 40 * 4, cu_new=INTS + 4, sel_pos=N * 4, ws=8 * MB)
AT = {name: (i + 1) * 16 * MB for i, name in enumerate(SIZES)}


@pytest.fixture(scope="module")
def lib():
    return B.load()


def _call(lib, name, **moved):
    at = {**AT, **moved}
    s, c = ctypes.byref(B.make_shape(HQ, HK, D, B.BF16)), ctypes.byref(B._PagedCache(at["k"], at["v"], PAGES, PAGE))
    p = ctypes.byref(B._PageTable(at["table"], at["ctx_len"], CTX, BATCH, 80))
    if name == "store":
        return lib.kvs_store_paged(s, c, p, at["cu_new"], at["sel_pos"], N, at["k_new"], at["v_new"], at["mass"], CTX, None)
    if name == "attention":
        return lib.kvs_attention_paged(s, c, p, at["cu_new"], at["sel_pos"], N, at["q"], 0.1, 0, 0, at["out"], at["lse_out"], at["ws"], 8 * MB, None)
    if name == "mass":
        return lib.kvs_mass_paged(s, c, p, at["cu_new"], at["sel_pos"], N, at["q"], at["lse"], 0.1, 0, 0, 1.0, at["mass"], at["mass_out"], CTX, at["ws"], 8 * MB, None)
    return lib.kvs_evict_paged(s, c, p, at["keep"], 500, 0, 0, at["mass"], CTX, at["new_table"], 40, at["kept"], at["new_len"], at["new_mass"], at["ws"], 8 * MB, None)


def _refused(lib, name, written, read):
    """`read` is moved over the first and over the last bytes of `written`, to 16-byte boundaries."""
    first, last = AT[written] - (SIZES[read] - 1) // 16 * 16, AT[written] + (SIZES[written] - 1) // 16 * 16
    for at in (first, AT[written], last):
        assert _call(lib, name, **{read: at}) == B.EINVAL, (written, read)
        text = lib.kvs_last_error()
        assert b"overlaps" in text and b"kvs_" + name.encode() + b"_paged" in text, text


@pytest.mark.parametrize("read", ["k_new", "v_new", "table", "ctx_len", "cu_new", "sel_pos"])
@pytest.mark.parametrize("written", ["k", "v", "mass"])
def test_store(lib, written, read):
    _refused(lib, "store", written, read)


@pytest.mark.parametrize("pool", ["k", "v"])
def test_store_mass_in_the_cache(lib, pool):
    _refused(lib, "store", pool, "mass")


@pytest.mark.parametrize("read", ["q", "k", "v", "table", "ctx_len", "cu_new", "sel_pos"])
@pytest.mark.parametrize("written", ["out", "lse_out"])
def test_attention(lib, written, read):
    _refused(lib, "attention", written, read)


def test_attention_outputs_over_each_other(lib):
    _refused(lib, "attention", "out", "lse_out")


@pytest.mark.parametrize("read", ["q", "lse", "mass", "k", "v", "table", "ctx_len", "cu_new", "sel_pos"])
def test_mass(lib, read):
    if read != "mass":                                       # (mass may be mass_out itself)
        _refused(lib, "mass", "mass_out", read)
    for at in (AT["mass_out"] - (SIZES[read] - 1) // 16 * 16, AT["mass_out"] + 16, AT["mass_out"] + SIZES["mass_out"] - 16):
        assert _call(lib, "mass", **{read: at}) == B.EINVAL and b"overlaps" in lib.kvs_last_error()


@pytest.mark.parametrize("read", ["mass", "keep", "table", "ctx_len", "new_table"])
@pytest.mark.parametrize("written", ["k", "v", "kept", "new_len", "new_mass"])
def test_evict(lib, written, read):
    if (written, read) != ("new_len", "ctx_len"):
        _refused(lib, "evict", written, read)


@pytest.mark.parametrize("one,other", [("k", "kept"), ("v", "kept"), ("k", "new_mass"), ("v", "new_mass"), ("k", "new_len"), ("v", "new_len"), ("kept", "new_mass"), ("kept", "new_len"), ("new_mass", "new_len")])
def test_evict_outputs_over_each_other(lib, one, other):
    _refused(lib, "evict", one, other)


def test_evict_lengths_in_place(lib):
    """new_len may be ctx_len itself, and lie across it in no other way."""
    for by in (-12, -4, 4, 12):
        assert _call(lib, "evict", new_len=AT["ctx_len"] + by) == B.EINVAL and b"new_len overlaps ctx_len" in lib.kvs_last_error()
    assert _call(lib, "evict", new_len=AT["ctx_len"], kept=AT["mass"]) == B.EINVAL and b"kept overlaps mass" in lib.kvs_last_error()
    assert _call(lib, "evict", new_len=AT["ctx_len"], kept=AT["ctx_len"]) == B.EINVAL and b"kept overlaps ctx_len" in lib.kvs_last_error()
