"""Tables that hx_kv_evict refuses before it touches the GPU."""
import ctypes as C

from tests.test_serve_refusals import INVALID, SHAPE, lib, pool, seqs  # noqa: F401


def test_rows_of_more_positions_than_weights_are_added_to(lib):  # noqa: F811
    """As hx_kv_weigh refuses them; a budget may be as large as it will, but has to hold what is kept in any case."""
    lib, ctx = lib

    def call(max_pages, n_keep=4, first=1, last=1):
        return lib.hx_kv_evict(ctx, C.byref(pool()), C.byref(seqs(max_pages=max_pages)), 1, 4096, 4096, n_keep, first, last, None, None)
    assert call((1 << 26) + 1) == SHAPE and call((1 << 27) - 1) == SHAPE and call(1 << 27) == SHAPE
    assert call((1 << 26) + 1, n_keep=2 ** 31 - 1) == SHAPE and call(4, 2 ** 31 - 1, 2 ** 31 - 1, 1) == INVALID


def test_weights_of_tables(lib):  # noqa: F811
    """Weights that are not aligned are refused by every call over the tables; an eviction by others than the tables' own, which it would leave behind."""
    from tests.test_serve_refusals import entry_points
    lib, ctx = lib
    assert list(entry_points(lib, ctx, pool(), seqs(weight=4098))) == [INVALID] * 7

    def call(own, w):
        return lib.hx_kv_evict(ctx, C.byref(pool()), C.byref(seqs(weight=own)), 1, 4096, w, 4, 1, 1, None, None)
    assert call(8192, 4096) == INVALID and b"own" in lib.hx_last_error(ctx) and call(4096 + 2, 4096 + 2) == INVALID
