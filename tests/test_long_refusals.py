"""What the entry points for long contexts refuse before they touch the GPU."""
import ctypes as C

import pytest

from paper_2605_16637_amd import binding
from tests.test_serve_refusals import INVALID, SHAPE, attend_args, entry_points, lib, pool, seqs  # noqa: F401


def four(**over):
    return pool(**{**dict(dtype=binding.HX_E2M1, k_exp=4096, v_exp=4096), **over})


@pytest.mark.parametrize("over,code", [(dict(head_dim=80), SHAPE), (dict(head_dim=48), SHAPE), (dict(k_exp=None), INVALID), (dict(v_exp=None), INVALID),
                                       (dict(k_exp=4100), INVALID), (dict(k_scale=4096), INVALID), (dict(bounds=4104), INVALID),
                                       (dict(n_heads=65536, page_tokens=256, head_dim=256), SHAPE)])
def test_pools_of_4_bits_that_are_refused(lib, over, code):  # noqa: F811
    lib, ctx = lib
    assert list(entry_points(lib, ctx, four(**over), seqs())) == [code] * 7


def test_scales_of_32_numbers_are_for_4_bits(lib):  # noqa: F811
    lib, ctx = lib
    for over in (dict(k_exp=4096), dict(v_exp=4096), dict(dtype=binding.HX_E4M3, k_exp=4096, v_exp=4096)):
        assert list(entry_points(lib, ctx, pool(**over), seqs())) == [INVALID] * 7


def test_reads_that_are_refused(lib):  # noqa: F811
    lib, ctx = lib
    p, s, a = C.byref(four()), C.byref(seqs()), 4096
    st = C.c_int64(128), C.c_int64(64)
    read = lambda layer, n, n_tok, t, k, v, p=p, s=s: lib.hx_kv_read(ctx, p, layer, s, n, a, a, n_tok, t, k, v, *st, None)  # noqa: E731
    assert read(2, 1, 1, binding.HX_F32, a, a) == INVALID and read(-1, 1, 1, binding.HX_F32, a, a) == INVALID
    assert read(0, -1, 1, binding.HX_F32, a, a) == INVALID and read(0, 1, -1, binding.HX_F32, a, a) == INVALID
    assert read(0, 1, 1, binding.HX_E4M3, a, a) == INVALID and read(0, 1, 1, binding.HX_E2M1, a, a) == INVALID
    assert read(0, 1, 1, binding.HX_F32, None, a) == INVALID and read(0, 1, 1, binding.HX_F32, a, a + 2) == INVALID
    assert read(0, 0, 1, binding.HX_F32, None, None) == 0 and read(0, 1, 0, binding.HX_F32, None, None) == 0
    assert read(0, 1, 1, binding.HX_F32, a, a, p=None) == INVALID and read(0, 1, 1, binding.HX_F32, a, a, s=None) == INVALID
    assert lib.hx_kv_write(ctx, p, 0, s, 1, a, a, 1, binding.HX_E2M1, a, a, *st, None) == INVALID
    assert lib.hx_attend(ctx, p, 0, s, C.byref(attend_args(dtype=binding.HX_F32)), None) == INVALID
    assert lib.hx_attend(ctx, C.byref(four(head_dim=96)), 0, s, C.byref(attend_args()), None) == SHAPE


def test_bounds_that_are_refused(lib):  # noqa: F811
    lib, ctx = lib
    s, a = C.byref(seqs()), 4096
    bound = lambda p, layer=0, n=1, row=a: lib.hx_kv_bound(ctx, C.byref(p), layer, s, n, row, None, None)  # noqa: E731
    assert bound(pool()) == INVALID                                            # a pool without
    with_bounds = pool(bounds=4096)
    assert bound(with_bounds, layer=2) == INVALID and bound(with_bounds, layer=-2) == INVALID
    assert bound(with_bounds, n=-1) == INVALID and bound(with_bounds, row=None) == INVALID and bound(with_bounds, n=0, row=None) == 0
    assert bound(pool(bounds=4096 + 8)) == INVALID and bound(pool(bounds=4096, n_layers=60000), layer=-1, n=1 << 20) == SHAPE
    assert lib.hx_kv_bound(ctx, C.byref(with_bounds), 0, C.byref(seqs(n=0, table=None, len=None)), 1, a, None, None) == INVALID


@pytest.mark.parametrize("over,code", [
    (dict(n_pages=0), INVALID), (dict(n_pages=-1), INVALID), (dict(n_first=-1), INVALID), (dict(n_last=0), INVALID), (dict(n_first=3, n_last=2), INVALID),
    (dict(n_first=2 ** 31 - 1, n_last=2 ** 31 - 1), INVALID), (dict(n_pages=4097), SHAPE)])
def test_choices_that_are_refused(lib, over, code):  # noqa: F811
    lib, ctx = lib
    t = binding.hx_top(**{**dict(n_pages=4, n_first=1, n_last=1, chosen=None), **over})
    assert lib.hx_attend_top(ctx, C.byref(pool(bounds=4096)), 0, C.byref(seqs()), C.byref(attend_args()), C.byref(t), None) == code


def test_chosen_pages_with_other_arguments(lib):  # noqa: F811
    lib, ctx = lib
    t = C.byref(binding.hx_top(4, 1, 1, None))

    def call(p=pool(bounds=4096), layer=0, a=None, top=t, **over):
        return lib.hx_attend_top(ctx, C.byref(p), layer, C.byref(seqs()), C.byref(attend_args(**over)) if a is None else a, top, None)
    assert call(top=None) == INVALID and call(p=pool()) == INVALID and call(layer=2) == INVALID
    assert call(window=5) == INVALID and call(parent=4096) == INVALID and call(q=None) == INVALID and call(out=None) == INVALID
    assert call(n_heads=3) == SHAPE and call(dtype=binding.HX_F16) == INVALID and call(n_q=0) == 0 and call(scale=float("nan")) == INVALID
    assert call(p=pool(bounds=4096, head_dim=96)) == SHAPE


def test_structures_match_the_header(tmp_path):
    import os
    import subprocess
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    cls = binding.hx_top
    lines = ['#include <stdio.h>', '#include <stddef.h>', '#include "hx.h"', 'int main(void) {', 'printf("%zu\\n", sizeof(hx_top));']
    lines += [f'printf("%zu\\n", offsetof(hx_top, {f}));' for f, _ in cls._fields_]
    (tmp_path / "a.c").write_text("\n".join(lines + ["return 0; }"]))
    subprocess.check_call(["gcc", "-std=c99", "-I", os.path.join(root, "include"), "-o", str(tmp_path / "a"), str(tmp_path / "a.c")])
    got = [int(x) for x in subprocess.check_output([str(tmp_path / "a")], text=True).split()]
    assert got == [C.sizeof(cls)] + [getattr(cls, f).offset for f, _ in cls._fields_]


def test_weighing_that_is_refused(lib):  # noqa: F811
    lib, ctx = lib

    def call(p=pool(), layer=0, w=4096, **over):
        return lib.hx_kv_weigh(ctx, C.byref(p), layer, C.byref(seqs()), C.byref(attend_args(**{**dict(lse=4096, out=None), **over})), w, None)
    assert call(w=None) == INVALID and call(lse=None) == INVALID and call(w=4097) == INVALID and call(lse=4098) == INVALID
    assert call(layer=2) == INVALID and call(q=None) == INVALID and call(n_heads=3) == SHAPE and call(max_q=257, parent=4096) == SHAPE
    assert call(p=pool(head_dim=96)) == SHAPE and call(dtype=binding.HX_F16) == INVALID and call(n_q=0, lse=None, w=None) == 0
    assert lib.hx_kv_weigh(ctx, C.byref(pool()), 0, C.byref(seqs()), None, 4096, None) == INVALID


@pytest.mark.parametrize("n_keep,n_first,n_last,code", [(0, 0, 0, INVALID), (-1, 0, 0, INVALID), (4, -1, 0, INVALID), (4, 0, -1, INVALID), (4, 3, 2, INVALID),
                                                        (2 ** 31 - 1, 2 ** 31 - 1, 2 ** 31 - 1, INVALID)])
def test_budgets_that_are_refused(lib, n_keep, n_first, n_last, code):  # noqa: F811
    lib, ctx = lib
    assert lib.hx_kv_evict(ctx, C.byref(pool()), C.byref(seqs()), 1, 4096, 4096, n_keep, n_first, n_last, None, None) == code


def test_evictions_that_are_refused(lib):  # noqa: F811
    lib, ctx = lib
    call = lambda n=1, row=4096, w=4096, p=pool(), s=seqs(): lib.hx_kv_evict(ctx, C.byref(p), C.byref(s), n, row, w, 4, 1, 1, None, None)  # noqa: E731
    assert call(n=-1) == INVALID and call(row=None) == INVALID and call(w=None) == INVALID and call(w=4098) == INVALID
    assert call(n=0, row=None, w=None) == 0 and call(s=seqs(n=0, table=None, len=None)) == INVALID
    assert call(n=1 << 20, p=pool(n_layers=1000)) == SHAPE and call(p=pool(dtype=0)) == INVALID and call(s=seqs(len=None)) == INVALID
