"""The library's second build, in which paged attention can be sent to its kernel of many rows (256 a workgroup), which the estimate
takes only for calls of some size; and what the estimate takes, asked without a call."""
import contextlib
import ctypes

from paper_2503_16525_amd import binding as B
from paper_2503_16525_amd.build import LIB_BIGATTN_PATH

FAKE = 0x10000


@contextlib.contextmanager
def forced(pieces):
    """Calls go through the second build: to the kernel of many rows with so many pieces, or (0) as the shipped library has it."""
    saved = B.LIB_PATH, B._lib
    B.LIB_PATH, B._lib = LIB_BIGATTN_PATH, None
    try:
        lib = B.load(build_if_missing=False)
        lib.kvs_test_force_pieces.restype = None
        lib.kvs_test_force_pieces(pieces)
        yield lib
        lib.kvs_test_force_pieces(0)
    finally:
        B.LIB_PATH, B._lib = saved


def choice(lib, shape, page, batch, max_ctx, n_new, ragged=True, listed=False, scale=0.1, window=0, n_first=0, ws_bytes=None, n_pages=1 << 20):
    """-> (kernel of many rows, pieces, row tiles dealt)"""
    if ws_bytes is None:
        ws_bytes = lib.kvs_workspace_size(b"attention_paged", ctypes.byref(shape), batch, max_ctx, n_new)
    lib.kvs_test_choice.argtypes = [ctypes.c_void_p] * 5 + [ctypes.c_int64, ctypes.c_float, ctypes.c_int32, ctypes.c_int32, ctypes.c_size_t, ctypes.c_void_p]
    taken = (ctypes.c_int32 * 3)()
    cache, pages = B._PagedCache(FAKE, FAKE, n_pages, page), B._PageTable(FAKE, FAKE, max_ctx, batch, -(-max_ctx // page))
    rc = lib.kvs_test_choice(ctypes.addressof(shape), ctypes.addressof(cache), ctypes.addressof(pages), FAKE if ragged else None, FAKE if listed else None, n_new, scale, window, n_first,
                             ws_bytes, ctypes.addressof(taken))
    assert rc == B.OK, lib.kvs_last_error()
    return bool(taken[0]), taken[1], bool(taken[2])
