"""Which kernel kvs_attention_paged takes, and how it cuts the keys: asked of the library's second build, on the host (no GPU, no
tensor is read).  The calls here are of kinds that the estimate was fitted to; if it is fitted again, the tests of the kernel of many
rows have to reach it still."""
import pytest

import paged_many as M
from paper_2503_16525_amd import binding as B


def _choice(hq, hk, batch, ctx, n, forced=0, **kw):
    with M.forced(forced) as lib:
        return M.choice(lib, B.make_shape(hq, hk, kw.pop("d", 128), kw.pop("dtype", B.BF16)), 16, batch, ctx, n, ragged=n != batch, **kw)


def test_long_chunks_go_to_the_kernel_of_many_rows():
    assert _choice(32, 8, 1, 32768, 2048) == (True, 1, False)
    assert _choice(32, 8, 1, 8192, 8192, window=4096, n_first=4) == (True, 1, True)
    assert _choice(28, 4, 1, 6000, 6000) == (True, 1, True)
    taken = _choice(32, 8, 1, 16384, 256)
    assert taken[0] and taken[1] > 1 and not taken[2]
    taken = _choice(32, 8, 1, 3000, 600, listed=True)
    assert taken[0] and taken[1] > 1 and not taken[2]


@pytest.mark.parametrize("kw", [dict(dtype=B.F32), dict(d=64), dict(scale=-0.1), dict(scale=0.0), dict(scale=1e38), dict(ws_bytes=0)])
def test_what_the_kernel_of_many_rows_cannot_take(kw):
    assert not _choice(32, 8, 1, 32768, 2048, **kw)[0] and not _choice(32, 8, 1, 32768, 2048, forced=1, **kw)[0]


def test_single_tokens_do_not():
    for batch, ctx in ((1, 1), (1, 601), (1, 131072), (64, 16384), (300, 4000)):
        assert not _choice(32, 8, batch, ctx, batch)[0]
    assert _choice(32, 4, 1, 131072, 1)[1] > 1 and _choice(28, 4, 1, 100, 1)[1] == 1


def test_the_switch_is_the_second_builds_alone():
    assert not hasattr(B.load(), "kvs_test_force_pieces") and not hasattr(B.load(), "kvs_test_choice")
    with M.forced(3):
        pass
    assert _choice(8, 2, 1, 3000, 100, forced=3) == (True, 3, False)
    assert _choice(8, 2, 1, 3000, 100) == _choice(8, 2, 1, 3000, 100) and not _choice(8, 2, 1, 3000, 100)[0]


def test_pieces_that_are_not_made():
    """Fewer than eight tiles of 32 keys each, more than 32 of them, more workgroups than two a compute unit, more than a workspace holds."""
    assert not _choice(8, 2, 1, 400, 100, forced=3)[0]
    assert not _choice(8, 2, 1, 100000, 100, forced=33)[0]
    assert not _choice(32, 8, 1, 32768, 2048, forced=3)[0]
    assert not _choice(8, 2, 1, 3000, 100, forced=2, ws_bytes=1000)[0]
