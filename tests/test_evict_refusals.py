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
