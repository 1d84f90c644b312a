"""What the serving step's entry points refuse before they touch the GPU: arguments that cannot be meant.  The checks come before anything of the
context is used, so a block of zeros stands in for it and no GPU is needed."""
import ctypes as C

import pytest

from paper_2605_16637_amd import binding

INVALID, SHAPE = -1, -2


@pytest.fixture
def lib():
    lib = binding.load()
    block = C.create_string_buffer(1 << 16)
    lib_ctx = C.cast(block, C.c_void_p)
    lib_ctx.keep = block
    return lib, lib_ctx


def pool(**over):
    d = dict(n_layers=2, n_pages=8, n_heads=2, page_tokens=16, head_dim=64, dtype=binding.HX_BF16, k=4096, v=4096, ref=4096, k_scale=None, v_scale=None)
    return binding.hx_kv_pool(**{**d, **over})


def seqs(**over):
    return binding.hx_kv_seqs(**{**dict(n=4, max_pages=4, table=4096, len=4096), **over})


def attend_args(**over):
    d = dict(n=2, row=None, q_ptr=4096, n_q=2, max_q=1, max_len=64, n_heads=4, dtype=binding.HX_BF16, q=4096, q_token=256, q_head=64,
             out=4096, out_token=256, out_head=64, lse=None, scale=0.125, window=0, n_sink=0, parent=None)
    return binding.hx_attend_args(**{**d, **over})


BAD_POOL = [(None, INVALID), (dict(n_layers=0), INVALID), (dict(n_pages=-1), INVALID), (dict(n_heads=0), INVALID), (dict(head_dim=0), INVALID),
            (dict(head_dim=40), SHAPE), (dict(head_dim=2048), SHAPE), (dict(page_tokens=0), SHAPE), (dict(page_tokens=24), SHAPE),
            (dict(page_tokens=2048), SHAPE), (dict(dtype=0), INVALID), (dict(dtype=binding.HX_F32), INVALID), (dict(k=None), INVALID),
            (dict(ref=None), INVALID), (dict(k=4104), INVALID), (dict(k_scale=4096), INVALID), (dict(n_heads=1 << 20), SHAPE)]
BAD_SEQS = [(None, INVALID), (dict(n=-1), INVALID), (dict(max_pages=-1), INVALID), (dict(table=None), INVALID), (dict(len=None), INVALID),
            (dict(max_pages=1 << 28), SHAPE)]


def entry_points(lib, ctx, p, s):
    p, s = (None if x is None else C.byref(x) for x in (p, s))
    a = 4096
    yield lib.hx_kv_fork(ctx, p, s, 1, a, a, None, None)
    yield lib.hx_kv_grow(ctx, p, s, 1, a, a, None)
    yield lib.hx_kv_write(ctx, p, 0, s, 1, a, a, 1, binding.HX_F32, a, a, C.c_int64(128), C.c_int64(64), None)
    yield lib.hx_kv_keep(ctx, p, s, 1, a, a, a, a, 1, None)
    yield lib.hx_kv_free(ctx, p, s, 1, a, None, None, None)
    yield lib.hx_kv_compact(ctx, p, s, None, None, None)
    yield lib.hx_attend(ctx, p, 0, s, C.byref(attend_args()), None)


@pytest.mark.parametrize("over,code", BAD_POOL)
def test_pools_that_are_refused(lib, over, code):
    lib, ctx = lib
    assert list(entry_points(lib, ctx, None if over is None else pool(**over), seqs())) == [code] * 7
    assert lib.hx_last_error(ctx)


@pytest.mark.parametrize("over,code", BAD_SEQS)
def test_tables_that_are_refused(lib, over, code):
    lib, ctx = lib
    assert list(entry_points(lib, ctx, pool(), None if over is None else seqs(**over))) == [code] * 7


def test_arrays_and_sizes_of_the_page_calls(lib):
    lib, ctx = lib
    p, s, a = C.byref(pool()), C.byref(seqs()), 4096
    none = C.byref(seqs(n=0, table=None, len=None))
    st = C.c_int64(128), C.c_int64(64)
    assert lib.hx_kv_fork(ctx, p, s, -1, a, a, None, None) == INVALID
    assert lib.hx_kv_fork(ctx, p, s, 1, None, a, None, None) == INVALID
    assert lib.hx_kv_fork(ctx, p, s, 1, a, None, None, None) == INVALID
    assert lib.hx_kv_fork(ctx, p, s, 0, None, None, None, None) == 0
    assert lib.hx_kv_fork(ctx, p, none, 1, a, a, None, None) == INVALID
    assert lib.hx_kv_fork(ctx, p, s, 1 << 30, a, a, None, None) == SHAPE
    assert lib.hx_kv_grow(ctx, p, s, 1, a, None, None) == INVALID
    assert lib.hx_kv_free(ctx, p, s, 1, a, a, None, None) == INVALID
    assert lib.hx_kv_free(ctx, p, s, 1, None, None, None, None) == INVALID
    assert lib.hx_kv_keep(ctx, p, s, 1, a, a, a, None, 3, None) == INVALID
    assert lib.hx_kv_keep(ctx, p, s, 1, a, a, a, a, -3, None) == INVALID
    assert lib.hx_kv_keep(ctx, p, s, 1 << 30, a, a, a, a, 3, None) == SHAPE
    write = lambda layer, n_tok, t, k, v: lib.hx_kv_write(ctx, p, layer, s, 1, a, a, n_tok, t, k, v, *st, None)  # noqa: E731
    assert write(2, 1, binding.HX_F32, a, a) == INVALID
    assert write(-1, 1, binding.HX_F32, a, a) == INVALID
    assert write(0, -1, binding.HX_F32, a, a) == INVALID
    assert write(0, 1, binding.HX_E4M3, a, a) == INVALID
    assert write(0, 1, binding.HX_F32, None, a) == INVALID
    assert write(0, 1, binding.HX_F32, a + 2, a) == INVALID
    assert write(0, 0, binding.HX_F32, None, None) == 0


@pytest.mark.parametrize("over,code", [
    (dict(n=-1), INVALID), (dict(n_q=-1), INVALID), (dict(max_q=-1), INVALID), (dict(max_len=-1), INVALID), (dict(window=-1), INVALID),
    (dict(n_sink=-1), INVALID), (dict(dtype=binding.HX_F16), INVALID), (dict(dtype=binding.HX_F32), INVALID), (dict(n_heads=3), SHAPE),
    (dict(n_heads=0), SHAPE), (dict(max_q=257, parent=4096), SHAPE), (dict(scale=float("inf")), INVALID), (dict(q=None), INVALID),
    (dict(out=None), INVALID), (dict(q_ptr=None), INVALID), (dict(q=4097), INVALID), (dict(max_q=1 << 30), SHAPE), (dict(n_q=0), 0), (dict(n=0), 0)])
def test_attention_that_is_refused(lib, over, code):
    lib, ctx = lib
    assert lib.hx_attend(ctx, C.byref(pool()), 0, C.byref(seqs()), C.byref(attend_args(**over)), None) == code


def test_attention_over_layers_and_heads_that_are_not_there(lib):
    lib, ctx = lib
    args = C.byref(attend_args())
    assert lib.hx_attend(ctx, C.byref(pool()), 2, C.byref(seqs()), args, None) == INVALID
    assert lib.hx_attend(ctx, C.byref(pool()), -1, C.byref(seqs()), args, None) == INVALID
    assert lib.hx_attend(ctx, C.byref(pool(head_dim=96)), 0, C.byref(seqs()), args, None) == SHAPE
    assert lib.hx_attend(ctx, C.byref(pool()), 0, C.byref(seqs()), None, None) == INVALID


def test_scale_that_is_no_number(lib):
    lib, ctx = lib
    assert lib.hx_attend(ctx, C.byref(pool()), 0, C.byref(seqs()), C.byref(attend_args(scale=float("nan"))), None) == INVALID


def test_sampling_that_is_refused(lib):
    lib, ctx = lib
    a = 4096

    def call(n=2, v=100, t=binding.HX_F32, logits=a, u=a, token=a):
        return lib.hx_sample(ctx, n, v, t, logits, C.c_int64(100), None, None, None, None, u, token, None, None, None)
    assert call(n=-1) == INVALID and call(v=-1) == INVALID and call(v=0) == INVALID
    assert call(v=524289) == SHAPE and call(t=binding.HX_E4M3) == INVALID
    assert call(logits=None) == INVALID and call(u=None) == INVALID and call(token=None) == INVALID and call(logits=a + 2) == INVALID
    assert call(n=0, logits=None) == 0
    assert b"aligned" in (call(logits=a + 2) and lib.hx_last_error(ctx))


def test_pages_of_2_gib_and_more(lib):
    lib, ctx = lib
    big = pool(n_heads=65536, page_tokens=64, head_dim=256)
    assert list(entry_points(lib, ctx, big, seqs())) == [SHAPE] * 7


def test_calls_too_large_to_launch_and_rows_too_long(lib):
    """Launches count threads in 32 bits; nothing of such a call is begun."""
    lib, ctx = lib
    a = 4096
    big = C.byref(pool(n_layers=32)), C.byref(seqs())
    assert lib.hx_kv_fork(ctx, *big, 300000, a, a, None, None) == SHAPE                       # 65 workgroups of 256 each
    assert lib.hx_kv_keep(ctx, *big, 300000, a, a, a, a, 3, None) == SHAPE
    assert lib.hx_kv_free(ctx, *big, 1 << 24, a, None, None, None) == SHAPE
    assert lib.hx_sample(ctx, 1 << 22, 100, binding.HX_F32, a, C.c_int64(100), None, None, None, None, a, a, None, None, None) == SHAPE
    assert lib.hx_attend(ctx, C.byref(pool(page_tokens=1024)), 0, C.byref(seqs(max_pages=1 << 20)), C.byref(attend_args()), None) == SHAPE


def test_structures_match_the_header(tmp_path):
    import os
    import subprocess
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    structs = {n: getattr(binding, n) for n in ("hx_kv_pool", "hx_kv_seqs", "hx_attend_args")}
    lines = ['#include <stdio.h>', '#include <stddef.h>', '#include "hx.h"', 'int main(void) {']
    for name, cls in structs.items():
        lines.append(f'printf("%zu\\n", sizeof({name}));')
        lines += [f'printf("%zu\\n", offsetof({name}, {f}));' for f, _ in cls._fields_]
    (tmp_path / "a.c").write_text("\n".join(lines + ["return 0; }"]))
    subprocess.check_call(["gcc", "-std=c99", "-I", os.path.join(root, "include"), "-o", str(tmp_path / "a"), str(tmp_path / "a.c")])
    got = [int(x) for x in subprocess.check_output([str(tmp_path / "a")], text=True).split()]
    assert got == [x for cls in structs.values() for x in [C.sizeof(cls)] + [getattr(cls, f).offset for f, _ in cls._fields_]]
