"""Caches of 4 bits, and numbers read from caches of every type, against plain forms in whole numbers and 64 bits."""
import numpy as np
import pytest

from tests import long_helpers as lh
from tests import serve_helpers as sh

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    from paper_2605_16637_amd import binding
    c = binding.Context(0)
    yield c
    c.close()


def empty_pool(layers, pages, heads, T, dim, ref=None):
    import torch
    u8 = lambda *s: torch.full(s, 0x99, dtype=torch.uint8, device="cuda:0")  # noqa: E731
    return dict(k=u8(layers, pages, heads, T, dim // 2), v=u8(layers, pages, heads, T, dim // 2), k_exp=u8(layers, pages, heads, T, dim // 32),
                v_exp=u8(layers, pages, heads, T, dim // 32), ref=sh.i32(np.ones(pages) if ref is None else ref))


def write(ctx, pool, x, y, T, layer=0):
    """One row's tokens over all pages of the pool, in order."""
    n = x.shape[0]
    seqs = dict(table=sh.i32([range(-(-n // T))]), len=sh.i32([n]))
    ctx.hx_kv_write(pool, layer, seqs, sh.i32([0]), sh.i32([0, n]), x, y)
    assert lh.status(ctx) == 0
    return seqs


def held(pool, name, layer, n, T):
    """Codes and bytes of a row's tokens, [n, heads, ..]."""
    codes = lh.unpacked(pool[name][layer].cpu().numpy()).transpose(0, 2, 1, 3)
    byte = pool[name + "_exp"][layer].cpu().numpy().astype(np.int64).transpose(0, 2, 1, 3)
    return codes.reshape(-1, *codes.shape[2:])[:n], byte.reshape(-1, *byte.shape[2:])[:n]


@pytest.mark.parametrize("src", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("heads,dim,T", [(1, 32, 1), (3, 96, 8), (8, 128, 16), (2, 256, 64)])
@pytest.mark.parametrize("wide", [True, False])
def test_write_rounds_to_the_nearest_code(ctx, src, heads, dim, T, wide):
    import torch
    n = 3 * T + 1
    g = torch.Generator().manual_seed(dim)
    x = torch.randn(n, 2 * heads, dim + (0 if wide else 1), generator=g) * torch.exp(4 * torch.randn(n, 2 * heads, 1, generator=g))
    x[0, 0, :32] = torch.tensor([0, 0.25, 0.5, 0.75, 1, 1.25, 1.5, 1.75, 2, 2.5, 3, 3.5, 4, 5, 6, -0.0, -0.25, -0.75, -1.25, -1.75, -2.5, -3.5, -5, -6,
                                 0.2501, 0.7499, 1.2501, 1.7499, 2.501, 3.499, 4.999, 5.001])
    x[0, 1, :32] = 0.0                                                # nothing in a group
    x[1, 0, :32] = 2.0 ** torch.linspace(-40, 15, 32)                 # beyond the largest, and far below
    x[1, 1, :32] = 1e-8 * torch.randn(32, generator=g)                # below the least scale
    x[2, 0, :32] = torch.cat([torch.tensor([6.0]), torch.linspace(-6, 6, 31)])
    x[2, 1, :32] = torch.cat([torch.tensor([6.0 + 2.0 ** -5]), torch.linspace(-6, 6, 31)])
    x = x.to(sh.torch_type(src)).cuda()
    k, v = x[:, :heads, :dim], x[:, heads:, :dim]
    pool = empty_pool(2, -(-n // T), heads, T, dim)
    write(ctx, pool, k, v, T, layer=1)
    for name, y in (("k", k), ("v", v)):
        codes, byte = held(pool, name, 1, n, T)
        want, want_byte = lh.encode(lh.f64(y))
        assert np.array_equal(byte, want_byte) and np.array_equal(codes, want)
        assert bool((pool[name][0] == 0x99).all()) and bool((pool[name + "_exp"][0] == 0x99).all())       # the other layer is as it was


@pytest.mark.parametrize("src", ["f32", "bf16", "f16"])
def test_write_of_infinities_and_nan(ctx, src):
    import torch
    x = torch.randn(4, 1, 64, generator=torch.Generator().manual_seed(1))
    x[0, 0, 3], x[0, 0, 40], x[1, 0, 63], x[2, 0, 0], x[2, 0, 1] = float("inf"), float("nan"), -float("inf"), float("nan"), float("inf")
    x = x.to(sh.torch_type(src)).cuda()
    pool = empty_pool(1, 2, 1, 2, 64)
    seqs = write(ctx, pool, x, -x, 2)
    out = torch.zeros(2, 4, 1, 64, device="cuda:0")
    ctx.hx_kv_read(pool, 0, seqs, sh.i32([0]), sh.i32([0, 4]), out[0], out[1])
    k, v = out.cpu().numpy()[:, :, 0]
    top = 6 * 2.0 ** 13
    assert k[0, 3] == top and v[0, 3] == -top and np.isnan(k[0, 32:]).all() and np.isnan(v[0, 32:]).all()
    assert k[1, 63] == -top and not np.isnan(k[1]).any() and (k[1, 32:63] == 0).all()
    assert np.isnan(k[2, :32]).all() and not np.isnan(k[2, 32:]).any() and not np.isnan(k[3]).any()


@pytest.mark.parametrize("cache", ["bf16", "f16", "e4m3", "e2m1"])
@pytest.mark.parametrize("dst", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("wide", [True, False])
@pytest.mark.parametrize("dim,T", [(32, 1), (96, 8), (128, 32)])
def test_read_gives_what_the_cache_holds(ctx, cache, dst, wide, dim, T):
    import torch
    lens, heads = [2 * T + 1, 70, 1, 5 * T], 3
    c = lh.Cache(3, lens, T, heads, dim, cache, missing=[(1, 0), (3, 2)])
    rows, count = [2, 0, 3, 1, 1], [1, 0, 4 * T, 70, 5]                        # a sequence may be read twice
    ptr = np.concatenate([[0], np.cumsum(count)])
    total, t = int(ptr[-1]), sh.torch_type(dst)
    both = torch.full((2, total, heads + 1, dim if wide else dim + 1), 7.0, dtype=t, device="cuda:0")
    k, v = (x[:, :heads, :dim] if wide else x[:, 1:, 1:] for x in both)
    ctx.hx_kv_read(c.pool, 1, c.seqs, sh.i32(c.where[rows]), sh.i32(ptr), k, v)
    assert lh.status(ctx) == 0
    for name, x, got in (("k", c.k, k), ("v", c.v, v)):
        for j, i in enumerate(rows):
            want = torch.as_tensor(c.of(x, 1, i)[lens[i] - count[j]:]).float().to(t).double().numpy()       # 8 bits times a scale: rounded to 32 bits first
            assert np.array_equal(lh.f64(got)[ptr[j]:ptr[j + 1]], want)
    edge = both[:, :, heads] if wide else torch.cat([both[:, :, 0].flatten(1), both[:, :, :, 0].flatten(1)], 1)
    assert bool((edge == 7.0).all())


def test_read_of_entries_in_error(ctx):
    import torch
    c = lh.Cache(4, [20, 9], 8, 2, 64, "e2m1", garbage=False)
    r0, r1 = (int(x) for x in c.where)
    rows, count = [r0, 99, -1, r1, r1], [20, 3, 2, 10, 9]                      # longer than the row: the fourth
    ptr = np.concatenate([[0], np.cumsum(count)])
    k, v = torch.full((2, int(ptr[-1]) + 4, 2, 64), 7.0, device="cuda:0")
    seqs = dict(table=c.seqs["table"].clone(), len=c.seqs["len"])
    seqs["table"][r0, 1] = c.n_pages + 3                                       # no page of the pool
    ctx.hx_kv_read(c.pool, 0, seqs, sh.i32(rows), sh.i32(ptr), k, v)
    assert lh.status(ctx) == -6
    want = c.of(c.k, 0, 0)
    want[8:16] = 0
    assert np.array_equal(lh.f64(k)[:20], want) and np.array_equal(lh.f64(k)[35:44], c.of(c.k, 0, 1))
    assert bool((k[20:35] == 7).all()) and bool((v[44:] == 7).all())           # tokens of no entry: left as they were
    ctx.hx_kv_read(c.pool, 0, c.seqs, sh.i32([]), sh.i32([0]), k[:0], v[:0])
    assert lh.status(ctx) == 0


@pytest.mark.parametrize("type_", ["bf16", "f16"])
@pytest.mark.parametrize("group", [1, 40])
def test_every_code_and_scale_is_read_exactly(ctx, type_, group):
    """A query that sees one token gets its value: all 16 codes with all scales that are written, by both kernels; and NaN."""
    import torch
    dim, T = 64, 1
    scales = list(range(lh.LEAST, lh.MOST + 1)) + [lh.NAN_BYTE]
    n = len(scales)
    codes = np.tile(np.arange(16), (n, 1, 1, 1, 4))
    byte = np.array(scales)[:, None, None, None].repeat(2, -1)
    pool = dict(k=sh.dev(lh.packed(codes)[None].reshape(1, n, 1, T, 32)), v=sh.dev(lh.packed(codes)[None].reshape(1, n, 1, T, 32)),
                k_exp=sh.dev(np.full((1, n, 1, T, 2), 127, np.uint8)), v_exp=sh.dev(byte.astype(np.uint8).reshape(1, n, 1, T, 2)), ref=sh.i32(np.ones(n)))
    seqs = dict(table=sh.i32(np.arange(n)[:, None]), len=sh.i32(np.ones(n)))
    q = torch.randn(n, group, dim, generator=torch.Generator().manual_seed(0)).to(sh.torch_type(type_)).cuda()
    out = torch.zeros_like(q)
    ctx.hx_attend(pool, 0, seqs, sh.i32(range(n + 1)), q, out, max_q=1)
    assert lh.status(ctx) == 0
    want = np.broadcast_to(lh.decode(np.tile(np.arange(16), (n, 4)), np.array(scales)[:, None].repeat(2, 1))[:, None], (n, group, dim))
    assert np.array_equal(lh.f64(out), want, equal_nan=True)
    # and as keys: a score of one code alone, against a query of one place
    one = torch.zeros(n, group, dim, dtype=q.dtype, device="cuda:0")
    one[:, :, 13] = 1.0
    pool["k_exp"], pool["v_exp"] = pool["v_exp"], pool["k_exp"]
    lse = torch.zeros(n, group, device="cuda:0")
    ctx.hx_attend(pool, 0, seqs, sh.i32(range(n + 1)), one, out, max_q=1, scale=1.0, lse=lse)
    got, want = lh.f64(lse)[:-1], want[:-1, :, 13]
    assert (np.abs(got - want) <= 2.0 ** -22 * np.abs(want) + 2.0 ** -22).all()


def check(ctx, lens, nq, heads=2, group=2, dim=64, T=16, type_="bf16", window=0, sinks=0, parents=None, scale=None, missing=(), wide=True, seed=0):
    import torch
    c = lh.Cache(seed, lens, T, heads, dim, "e2m1", missing=missing)
    ptr = np.concatenate([[0], np.cumsum(nq)])
    total = int(ptr[-1])
    q = lh.queries(total, heads * group, dim, type_, seed, wide)
    out = torch.full_like(q, 7.0)
    lse = torch.full((total, heads * group), 7.0, device="cuda:0")
    par = None if parents is None else sh.i32(np.concatenate([np.asarray(p, np.int64) for p in parents]))
    ctx.hx_attend(c.pool, 1, c.seqs, sh.i32(ptr), q, out, max_q=max(nq), row=sh.i32(c.where), scale=scale, window=window, n_sink=sinks, parent=par, lse=lse)
    assert lh.status(ctx) == 0
    for i in range(len(lens)):
        see = sh.visible(lens[i], nq[i], None if parents is None else parents[i], window, sinks) & c.there(i)
        part = slice(ptr[i], ptr[i + 1])
        lh.compare(lh.f64(out)[part], lh.f64(lse)[part], lh.f64(q)[part], c.of(c.k, 1, i), c.of(c.v, 1, i), see,
                   dim ** -0.5 if scale is None else scale, group, type_)


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("type_", ["bf16", "f16"])
@pytest.mark.parametrize("T", [1, 8, 16, 64])
def test_one_query_each(ctx, dim, type_, T):
    lens = [1, 2, 15, 16, 17, 63, 64, 65, 130, 257, 700]
    check(ctx, lens, [1] * len(lens), dim=dim, type_=type_, T=T)


@pytest.mark.parametrize("heads,group", [(1, 1), (1, 7), (3, 1), (1, 16), (1, 17), (2, 33), (8, 4)])
@pytest.mark.parametrize("dim", [64, 128])
def test_head_layouts(ctx, heads, group, dim):
    check(ctx, [5, 90, 200], [1, 3, 2], heads=heads, group=group, dim=dim)


@pytest.mark.parametrize("window,sinks", [(0, 0), (1, 0), (17, 5), (64, 70), (65, 1), (500, 3)])
@pytest.mark.parametrize("T", [4, 32])
def test_windows_and_sinks(ctx, window, sinks, T):
    lens = [1, 40, 64, 129, 300, 411]
    check(ctx, lens, [1] * 6, window=window, sinks=sinks, T=T)
    check(ctx, lens, [1, 40, 9, 70, 150, 33], group=3, heads=1, window=window, sinks=sinks, T=T, seed=1)


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("type_", ["bf16", "f16"])
@pytest.mark.parametrize("rows,T", [(20, 16), (50, 8), (300, 16), (130, 64)])
def test_prompts(ctx, dim, type_, rows, T):
    check(ctx, [rows, rows + 1, 2 * rows + 77], [rows, rows - 3, rows], dim=dim, type_=type_, heads=1, group=2, T=T)


@pytest.mark.parametrize("rows", [1, 9, 40])
def test_long_contexts_are_divided_and_joined(ctx, rows):
    check(ctx, [4096, 3001], [rows, 1], heads=1, group=4, dim=128)


@pytest.mark.parametrize("n", [1, 8, 25, 200])
def test_trees(ctx, n):
    rng = np.random.default_rng(n)
    tree = lambda near: [int(rng.integers(max(-1, i - near), i)) for i in range(n)]  # noqa: E731
    check(ctx, [n, n + 1, n + 100], [n] * 3, heads=1, group=3, dim=128, parents=[tree(x) for x in (1, 4, 300)], window=40 if n == 25 else 0, sinks=2)


def test_pages_that_are_not_there_strides_and_scales(ctx):
    check(ctx, [40, 64, 300, 16], [1, 1, 60, 1], missing=[(0, 0), (1, 1), (2, 5), (3, 0)])
    check(ctx, [40, 64, 300, 16], [3, 62, 20, 1], wide=False, T=8)
    for scale in (0.0, -0.3, 2.0):
        check(ctx, [100, 50], [1, 40], scale=scale)


def test_many_small_weights_beside_a_large_one(ctx):
    """A weight of 1 beside 5999 of 2^-14.4 (scores 10 apart): thousands that sum to a quarter are not lost."""
    import torch
    n, dim, T = 6000, 64, 16
    pages = -(-n // T)
    k, v = torch.zeros(n, 1, dim, device="cuda:0"), torch.ones(n, 1, dim, device="cuda:0")
    k[0, 0, 0], v[0] = 2.0, -1.0
    pool = empty_pool(1, pages, 1, T, dim)
    seqs = write(ctx, pool, k, v, T)
    for type_ in ("bf16", "f16"):
        q = torch.zeros(1, 2, dim, dtype=sh.torch_type(type_), device="cuda:0")
        q[:, :, 0] = 5.0
        out = torch.zeros_like(q)
        ctx.hx_attend(pool, 0, seqs, sh.i32([0, 1]), q, out, max_q=1, scale=1.0)
        small = (n - 1) * np.exp(-10.0)
        want = (small - 1) / (small + 1)
        assert (np.abs(lh.f64(out) - want) <= 2 * sh.HALF_STEP[type_] * abs(want) + n * 2.0 ** -24).all()


# ---- pages ------------------------------------------------------------------------------------------------------------

def moved_cache(seed, lens, T, heads, dim, layers=2, rows=None, spare=6):
    """A cache as its codes and bytes, whose pages the plain rules move: `numbers` of a token are its codes, then its bytes."""
    rng = np.random.default_rng(seed)
    need = [-(-n // T) for n in lens]
    rows = len(lens) + 4 if rows is None else rows
    n_pages = sum(need) + spare
    order = rng.permutation(n_pages)
    table, ref, at = np.full((rows, max(need + [1]) + 2), -1), np.zeros(n_pages, np.int64), 0
    for i, k in enumerate(need):
        table[i, :k] = order[at:at + k]
        at += k
    ref[order[:at]] = 1
    length = np.zeros(rows, np.int64)
    length[:len(lens)] = lens
    half = dim // 2
    k, v = (rng.integers(0, 256, (layers, n_pages, heads, T, half + dim // 32)) for _ in range(2))
    model = sh.Pages(table, length, ref, k, v, T)
    u8 = lambda x: sh.dev(x.astype(np.uint8))  # noqa: E731
    pool = dict(k=u8(k[..., :half]), v=u8(v[..., :half]), k_exp=u8(k[..., half:]), v_exp=u8(v[..., half:]), ref=sh.i32(ref))
    return model, pool, dict(table=sh.i32(table), len=sh.i32(length))


def same(model, pool, seqs):
    half = pool["k"].shape[-1]
    assert np.array_equal(seqs["len"].cpu().numpy(), model.len) and np.array_equal(seqs["table"].cpu().numpy(), model.table)
    assert np.array_equal(pool["ref"].cpu().numpy(), model.ref)
    for name, x in (("k", model.k), ("v", model.v)):
        assert np.array_equal(pool[name].cpu().numpy(), x[..., :half]) and np.array_equal(pool[name + "_exp"].cpu().numpy(), x[..., half:])


@pytest.mark.parametrize("T", [1, 2, 8, 64])
@pytest.mark.parametrize("heads,dim", [(1, 32), (3, 64), (2, 96), (2, 128), (1, 512)])
def test_pages_of_4_bits_move_with_their_scales(ctx, T, heads, dim):
    lens = [5 * T + 3, 130, T + 1, 40]
    model, pool, seqs = moved_cache(T + dim, lens, T, heads, dim, rows=12)
    model.fork([0, 1, 1], [8, 9, 10], [5 * T + 3, 77, 2])
    ctx.hx_kv_fork(pool, seqs, sh.i32([0, 1, 1]), sh.i32([8, 9, 10]), sh.i32([5 * T + 3, 77, 2]))
    assert lh.status(ctx) == 0
    same(model, pool, seqs)
    row, drafts, kept = [3, 2], [40, 1], [[1, 2, 5, 17, 39], []]
    model.keep(row, drafts, kept)
    ends = np.concatenate([[0], np.cumsum([len(k) for k in kept])])
    ctx.hx_kv_keep(pool, seqs, sh.i32(row), sh.i32(drafts), sh.i32(ends), sh.i32(sum(kept, [])))
    assert lh.status(ctx) == 0
    same(model, pool, seqs)
    model.give([1])
    ctx.hx_kv_free(pool, seqs, sh.i32([1]))
    used, moved = model.compact()
    n_used = sh.i32([0])
    ctx.hx_kv_compact(pool, seqs, n_used=n_used)
    assert lh.status(ctx) == 0 and int(n_used) == used
    same(model, pool, seqs)


def test_write_of_4_bits_to_rows_in_error(ctx):
    """A row listed twice, a shared page, more tokens than the row has, a page that is not there: nothing of theirs is written."""
    import torch
    model, pool, seqs = moved_cache(5, [20, 9, 31, 16], 8, 2, 64)
    model.table[3, 1] = -1
    seqs["table"][3, 1] = -1
    pool["ref"][int(model.table[1, 1])] = model.ref[model.table[1, 1]] = 2
    count = [5, 2, 3, 40, 1]
    rows = [0, 0, 1, 2, 3]                                                     # 1: its last page is another's too, in which all of its three lie but two
    ptr = np.concatenate([[0], np.cumsum(count)])
    x = torch.randn(2, int(ptr[-1]), 2, 64, generator=torch.Generator().manual_seed(2)).cuda()
    ctx.hx_kv_write(pool, 0, seqs, sh.i32(rows), sh.i32(ptr), x[0], x[1])
    assert lh.status(ctx) == -6
    for name, y, m in (("k", x[0], model.k), ("v", x[1], model.v)):
        codes, byte = lh.encode(lh.f64(y))
        line = np.concatenate([lh.packed(codes), byte.astype(np.uint8)], -1)
        for j in range(5):
            m[0, model.table[0, (15 + j) // 8], :, (15 + j) % 8] = line[j]
        for j in range(2):                                                     # positions 6 and 7 of row 1, in its first page
            m[0, model.table[1, 0], :, 6 + j] = line[7 + j]
    same(model, pool, seqs)


def test_captured_and_on_another_stream(ctx):
    """Write, read and attend on a stream of their own, captured and replayed with other inputs between eager calls."""
    import torch
    T, heads, dim, n = 16, 2, 64, 50
    pool, seqs = empty_pool(1, 4, heads, T, dim), dict(table=sh.i32([range(4)]), len=sh.i32([n]))
    x, y = torch.zeros(2, n, heads, dim, device="cuda:0")
    q = torch.randn(3, heads * 2, dim, device="cuda:0", generator=torch.Generator("cuda:0").manual_seed(1)).bfloat16()
    out, k, v = torch.zeros_like(q), torch.zeros(n, heads, dim, device="cuda:0"), torch.zeros(n, heads, dim, device="cuda:0")
    row, ptr, q_ptr = sh.i32([0]), sh.i32([0, n]), sh.i32([0, 3])

    def calls(s):
        ctx.hx_kv_write(pool, 0, seqs, row, ptr, x, y, stream=s)
        ctx.hx_kv_read(pool, 0, seqs, row, ptr, k, v, stream=s)
        ctx.hx_attend(pool, 0, seqs, q_ptr, q, out, max_q=3, row=row, stream=s)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    calls(s)
    s.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        calls(s)
    for seed in range(3):
        g = torch.Generator("cuda:0").manual_seed(seed)
        x.copy_(torch.randn(n, heads, dim, device="cuda:0", generator=g))
        y.copy_(torch.randn(n, heads, dim, device="cuda:0", generator=g))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        a = [t.clone() for t in (k, v, out)]
        for t in (k, v, out):
            t.zero_()
        calls(None)
        torch.cuda.synchronize()
        assert all(torch.equal(p, t) for p, t in zip(a, (k, v, out)))
        assert np.array_equal(lh.f64(k), lh.decode(*lh.encode(lh.f64(x))))


@pytest.mark.parametrize("pages,entries", [(0, 0), (0, 3), (4, 0), (4, 3)])
@pytest.mark.parametrize("rows", [1, 40])
def test_queries_of_rows_that_hold_nothing(ctx, pages, entries, rows):
    """Pools without pages, tables without entries, rows that the tables lack: zeros, and no page is read."""
    import torch
    heads, group, dim, T = 2, 2, 64, 16
    pool = dict(empty_pool(1, pages, heads, T, dim), page_tokens=T)
    seqs = dict(table=torch.full((2, entries), -1, dtype=torch.int32, device="cuda:0"), len=sh.i32([0, 0]))
    q = torch.randn(2 * rows, heads * group, dim, device="cuda:0").bfloat16()
    out, lse = torch.full_like(q, 7.0), torch.full((2 * rows, heads * group), 7.0, device="cuda:0")
    ctx.hx_attend(pool, 0, seqs, sh.i32([0, rows, 2 * rows]), q, out, max_q=rows, row=sh.i32([1, 2]), max_len=max(1, entries * T), lse=lse)
    assert lh.status(ctx) == -6                                                # more queries than tokens, and no row 2
    assert (out == 0).all() and torch.isneginf(lse).all()
    weight = torch.full((2, entries * T), 7.0, device="cuda:0")
    if entries:
        ctx.hx_kv_weigh(pool, 0, seqs, sh.i32([0, rows, 2 * rows]), q, lse, weight, max_q=rows, row=sh.i32([1, 2]), max_len=entries * T)
        assert lh.status(ctx) == -6 and (weight == 7).all()
