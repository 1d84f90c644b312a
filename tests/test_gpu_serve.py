"""The serving step's operators against their plain forms in whole numbers and 64 bits."""
import math

import numpy as np
import pytest

from tests import serve_helpers as sh

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    from paper_2605_16637_amd import binding
    c = binding.Context(0)
    yield c
    c.close()


# ---- pages -------------------------------------------------------------------------------------------------------------

def make_cache(seed, lens, T, layers=2, heads=2, dim=32, rows=None, max_pages=None, spare=6, type_="bf16"):
    """A cache whose first rows hold sequences of these lengths on pages drawn at random; numbers that every type holds exactly."""
    import torch
    rng = np.random.default_rng(seed)
    need = [-(-n // T) for n in lens]
    rows = len(lens) + 4 if rows is None else rows
    max_pages = max(need + [1]) + 2 if max_pages is None else max_pages
    n_pages = sum(need) + spare
    order = rng.permutation(n_pages)
    table, ref, at = np.full((rows, max_pages), -1), np.zeros(n_pages, np.int64), 0
    for i, k in enumerate(need):
        table[i, :k] = order[at:at + k]
        at += k
    ref[order[:at]] = 1
    length = np.zeros(rows, np.int64)
    length[:len(lens)] = lens
    k, v = (rng.integers(-15, 16, (layers, n_pages, heads, T, dim)).astype(np.float64) for _ in range(2))
    model = sh.Pages(table, length, ref, k, v, T)
    t = sh.torch_type(type_)
    pool = dict(k=sh.dev(k, torch.float32).to(t), v=sh.dev(v, torch.float32).to(t), ref=sh.i32(ref), page_tokens=T)
    return model, pool, dict(table=sh.i32(table), len=sh.i32(length))


def same(model, pool, seqs, numbers=True):
    assert np.array_equal(seqs["len"].cpu().numpy(), model.len)
    assert np.array_equal(seqs["table"].cpu().numpy(), model.table)
    assert np.array_equal(pool["ref"].cpu().numpy(), model.ref)
    if numbers:
        assert np.array_equal(pool["k"].float().cpu().numpy(), model.k) and np.array_equal(pool["v"].float().cpu().numpy(), model.v)


def status(ctx):
    from paper_2605_16637_amd import binding
    try:
        ctx.hx_stream_status()
    except binding.HxError as e:
        return e.code
    return 0


@pytest.mark.parametrize("T", [1, 4, 16, 64])
@pytest.mark.parametrize("type_", ["bf16", "f16", "e4m3"])
def test_fork_shares_pages_and_copies_the_tail(ctx, T, type_):
    lens = [0, 1, T - 1 if T > 1 else 2, T, T + 1, 5 * T + 3, 130]
    model, pool, seqs = make_cache(1, lens, T, rows=20, type_=type_)
    src, dst = [5, 5, 6, 1, 0, 3, 4], [12, 7, 19, 8, 9, 10, 11]
    assert model.fork(src, dst) == set()
    ctx.hx_kv_fork(pool, seqs, sh.i32(src), sh.i32(dst))
    assert status(ctx) == 0
    same(model, pool, seqs)
    # parts of a sequence, among them none of it and whole pages of it
    src, dst, n_tok = [5, 6, 6, 5], [13, 14, 15, 16], [2, 0, min(130, 2 * T), 5 * T]
    assert model.fork(src, dst, n_tok) == set()
    ctx.hx_kv_fork(pool, seqs, sh.i32(src), sh.i32(dst), sh.i32(n_tok))
    assert status(ctx) == 0
    same(model, pool, seqs)


def test_fork_of_rows_in_error_leaves_them(ctx):
    model, pool, seqs = make_cache(2, [20, 33, 7], 8, rows=10, spare=2)
    src, dst, n_tok = [0, 1, 0, 99, 1, -1, 0, 1, 2], [4, 1, 4, 5, -3, 6, 7, 8, 9], [20, 33, 5, 1, 1, 1, 21, 33, 7]
    #          a copy, onto itself, twice, out of range (3), longer than its source, a copy, no page left
    assert model.fork(src, dst, n_tok) == {-6, -4}
    ctx.hx_kv_fork(pool, seqs, sh.i32(src), sh.i32(dst), sh.i32(n_tok))
    assert status(ctx) in (-6, -4)
    same(model, pool, seqs)
    assert status(ctx) == 0


def test_fork_of_a_source_that_gave_pages_back(ctx):
    model, pool, seqs = make_cache(3, [45, 40], 8, rows=6)
    model.give([0, 1], [8, 0], [32, 40])
    ctx.hx_kv_free(pool, seqs, sh.i32([0, 1]), sh.i32([8, 0]), sh.i32([32, 40]))
    model.fork([0, 1, 1], [2, 3, 4], [45, 40, 37])       # the last one's tail lies in a page that is not there
    ctx.hx_kv_fork(pool, seqs, sh.i32([0, 1, 1]), sh.i32([2, 3, 4]), sh.i32([45, 40, 37]))
    assert status(ctx) == 0
    same(model, pool, seqs)


@pytest.mark.parametrize("T,n", [(1, 5), (16, 7), (16, 1500), (64, 300)])
def test_grow_takes_the_lowest_free_pages_in_order(ctx, T, n):
    rng = np.random.default_rng(T + n)
    lens = rng.integers(0, 3 * T + 2, n).tolist()
    model, pool, seqs = make_cache(4, lens, T, layers=1, heads=1, dim=16, rows=n + 3, max_pages=9, spare=6 * n)
    row = rng.permutation(n)
    new = rng.integers(0, 3 * T + 1, n)
    assert model.grow(row, new) == set()
    ctx.hx_kv_grow(pool, seqs, sh.i32(row), sh.i32(new))
    assert status(ctx) == 0
    same(model, pool, seqs, numbers=False)


def test_grow_beyond_the_pool_and_rows_in_error(ctx):
    model, pool, seqs = make_cache(5, [10, 8, 3, 16], 8, rows=8, max_pages=6, spare=3)
    row, new = [0, 7, 0, 9, 1, 2, 3, 5, 4], [7, 4, 1, 1, 41, 2, 30, 3, 0]
    assert model.grow(row, new) == {-6, -4}
    ctx.hx_kv_grow(pool, seqs, sh.i32(row), sh.i32(new))
    assert status(ctx) in (-6, -4)
    same(model, pool, seqs, numbers=False)


@pytest.mark.parametrize("src", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("type_", ["bf16", "f16", "e4m3"])
@pytest.mark.parametrize("wide", [True, False])
def test_write_rounds_to_the_pools_type(ctx, src, type_, wide):
    import torch
    T, heads, dim = 8, 3, 48
    model, pool, seqs = make_cache(6, [20, 9, 0, 31], T, heads=heads, dim=dim, type_=type_)
    row, ptr = [3, 0, 1], [0, 5, 5, 14]
    g = torch.Generator().manual_seed(7)
    x = (torch.randn(14, 2 * heads, dim + (0 if wide else 1), generator=g) * 3)
    x[3, 0, :6] = torch.tensor([0.0, -0.0, 1e-5, 60000.0, -1000.0, 448.0])
    x = x.to(sh.torch_type(src)).cuda()
    k, v = x[:, :heads, :dim], x[:, heads:, :dim]
    scale = torch.tensor([[0.5, 2.0, 0.07], [1.0, 0.3, 11.0]], device="cuda:0")
    if type_ == "e4m3":
        pool["k_scale"], pool["v_scale"] = scale, scale * 3

    def stored(y, s):
        y = y.float()
        if type_ == "e4m3":
            y = (y / s[None, :, None]).clamp(-448, 448)
        return y.to(sh.torch_type(type_)).float().cpu().numpy().astype(np.float64)
    model.write(1, row, ptr, stored(k, scale[1]), stored(v, 3 * scale[1]))
    ctx.hx_kv_write(pool, 1, seqs, sh.i32(row), sh.i32(ptr), k, v)
    assert status(ctx) == 0
    same(model, pool, seqs)


@pytest.mark.parametrize("src", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("type_", ["bf16", "f16", "e4m3"])
def test_write_of_infinities_and_nan(ctx, src, type_):
    import torch
    model, pool, seqs = make_cache(16, [8], 8, layers=1, heads=1, dim=16, type_=type_)
    x = torch.zeros(8, 1, 16)
    x[0, 0, :6] = torch.tensor([float("inf"), -float("inf"), float("nan"), 1.0, -1.0, 0.0])
    x[1, 0, 5], x[7, 0, 15], x[7, 0, 3] = float("nan"), -float("inf"), 2.0
    x = x.to(sh.torch_type(src)).cuda()
    x[2, 0, 4] = -x[0, 0, 2]
    ctx.hx_kv_write(pool, 0, seqs, sh.i32([0]), sh.i32([0, 8]), x, -x)
    assert status(ctx) == 0
    page = int(model.table[0, 0])
    for mine, given in ((pool["k"], x), (pool["v"], -x)):
        want = given.float()
        if type_ == "e4m3":
            want = torch.where(want.isnan(), want, want.clamp(-448, 448))
        got = mine[0, page, 0].float()
        assert torch.equal(got.isnan(), want[:, 0].isnan()) and torch.equal(got.nan_to_num(9, 8, -8), want[:, 0].nan_to_num(9, 8, -8))


def test_write_does_not_touch_what_others_hold_or_what_is_not_there(ctx):
    import torch
    model, pool, seqs = make_cache(8, [16, 12], 8, heads=1, dim=16)
    model.fork([0], [3])
    ctx.hx_kv_fork(pool, seqs, sh.i32([0]), sh.i32([3]))
    x = torch.ones(4, 1, 16, dtype=torch.bfloat16, device="cuda:0")
    for row, ptr in (([0], [0, 2]), ([9], [0, 2]), ([1], [0, 13]), ([1], [3, 4])):
        ctx.hx_kv_write(pool, 0, seqs, sh.i32(row), sh.i32(ptr), x[:1].expand(4, 1, 16).contiguous()[:4] if ptr[1] <= 4 else x.repeat(4, 1, 1)[:13], x if ptr[1] <= 4 else x.repeat(4, 1, 1)[:13])
        assert status(ctx) == -6
    model.write(0, [1], [0, 12], np.ones((12, 1, 16)), np.ones((12, 1, 16)))      # of 13 tokens the first lies before the row's
    pool_k = pool["k"].float().cpu().numpy()
    assert np.array_equal(pool_k[:, model.table[0, :2]], model.k[:, model.table[0, :2]])


@pytest.mark.parametrize("heads,dim", [(1, 16), (2, 48), (8, 128)])
@pytest.mark.parametrize("n", [2, 9, 200])
def test_write_of_rows_listed_twice(ctx, n, heads, dim):
    """Of a row's entries the first is written, with other tokens in the others, which are as many or more or fewer; the rest of the call is carried out."""
    import torch
    rng = np.random.default_rng(n + dim)
    T, rows = 4, max(2, n // 3)
    lens = (8 + rng.integers(0, 20, rows)).tolist()
    model, pool, seqs = make_cache(22, lens, T, layers=1, heads=heads, dim=dim)
    row = rng.integers(0, rows, n)
    row[n // 2] = row[0]
    new = rng.integers(0, 9, n)
    new[0] = new[n // 2] = 5
    ptr = np.concatenate([[0], np.cumsum(new)])
    x = torch.as_tensor(rng.integers(-15, 16, (int(ptr[-1]), 2 * heads, dim))).to(torch.bfloat16).cuda()
    k, v = x[:, :heads], x[:, heads:]
    kf, vf = (y.float().cpu().numpy().astype(np.float64) for y in (k, v))
    for i in range(n):
        if row[i] not in row[:i]:
            model.write(0, [row[i]], [0, int(new[i])], kf[ptr[i]:ptr[i + 1]], vf[ptr[i]:ptr[i + 1]])
    ctx.hx_kv_write(pool, 0, seqs, sh.i32(row), sh.i32(ptr), k, v)
    assert status(ctx) == -6
    same(model, pool, seqs)


def test_write_of_entries_in_error_writes_none_of_their_tokens(ctx):
    import torch
    model, pool, seqs = make_cache(23, [12, 20, 9, 16], 8, heads=2, dim=32)
    x = torch.ones(40, 2, 32, dtype=torch.bfloat16, device="cuda:0")
    one = np.ones((40, 2, 32))
    # more tokens than the row has; an end beyond the tokens given; a row that is not there: the others are written
    for row, ptr, fine in (([0, 1], [0, 13, 17], [1]), ([2, 0], [0, 3, 41], [0]), ([9, 3, -1], [0, 4, 8, 10], [1])):
        ctx.hx_kv_write(pool, 0, seqs, sh.i32(row), sh.i32(ptr), x, x)
        assert status(ctx) == -6
        for i in fine:
            model.write(0, [row[i]], [0, ptr[i + 1] - ptr[i]], one[:ptr[i + 1] - ptr[i]], one[:ptr[i + 1] - ptr[i]])
        same(model, pool, seqs)


@pytest.mark.parametrize("T", [1, 8, 32])
@pytest.mark.parametrize("type_", ["bf16", "e4m3"])
def test_keep_moves_the_accepted_together(ctx, T, type_):
    rng = np.random.default_rng(T)
    lens = [40, 33, 64, 5, 71]
    model, pool, seqs = make_cache(9, lens, T, layers=3, heads=3, dim=48, type_=type_)
    row, drafts = [4, 0, 3, 2, 1], [17, 40, 5, 12, 0]
    kept = [sorted(rng.permutation(17)[:6].tolist()), list(range(40)), [], [0, 1, 11], []]
    ptr = np.concatenate([[0], np.cumsum([len(x) for x in kept])])
    model.keep(row, drafts, kept)
    ctx.hx_kv_keep(pool, seqs, sh.i32(row), sh.i32(drafts), sh.i32(ptr), sh.i32(sum(kept, [])))
    assert status(ctx) == 0
    same(model, pool, seqs)


def test_keep_of_long_lists(ctx):
    rng = np.random.default_rng(3)
    lens = [700, 420, 900]
    model, pool, seqs = make_cache(19, lens, 16, layers=2, heads=2, dim=16)
    drafts = [600, 400, 900]
    kept = [sorted(rng.permutation(n)[:m].tolist()) for n, m in ((600, 391), (400, 129), (900, 128))]
    ptr = np.concatenate([[0], np.cumsum([len(x) for x in kept])])
    model.keep([0, 1, 2], drafts, kept)
    ctx.hx_kv_keep(pool, seqs, sh.i32([0, 1, 2]), sh.i32(drafts), sh.i32(ptr), sh.i32(sum(kept, [])))
    assert status(ctx) == 0
    same(model, pool, seqs)


def test_keep_of_tokens_whose_pages_are_gone(ctx):
    """What stays where it is needs no page; a pool of no pages has none to look at."""
    import torch
    x = torch.zeros(1, 0, 1, 8, 16, dtype=torch.bfloat16, device="cuda:0")
    seqs = dict(table=sh.i32([[-1, -1], [-1, -1]]), len=sh.i32([9, 4]))
    ctx.hx_kv_keep(dict(k=x, v=x, ref=sh.i32([])), seqs, sh.i32([0, 1]), sh.i32([5, 2]), sh.i32([0, 3, 4]), sh.i32([0, 1, 2, 0]))
    assert status(ctx) == 0
    assert seqs["len"].tolist() == [7, 3]


@pytest.mark.parametrize("n", [1, 3, 64, 65, 300, 5000])
@pytest.mark.parametrize("dim,heads", [(16, 1), (128, 4)])
def test_write_of_many_sequences(ctx, n, dim, heads):
    import torch
    rng = np.random.default_rng(n)
    T = 4
    lens = rng.integers(0, 3 * T, n)
    model, pool, seqs = make_cache(17, lens.tolist(), T, layers=1, heads=heads, dim=dim, rows=n + 1)
    row = rng.permutation(n)
    new = np.where(rng.random(n) < 0.5, 0, rng.integers(0, lens[row] + 1))
    ptr = np.concatenate([[0], np.cumsum(new)])
    x = torch.as_tensor(rng.integers(-15, 16, (int(ptr[-1]), 2 * heads, dim))).to(torch.bfloat16).cuda()
    k, v = x[:, :heads], x[:, heads:]
    model.write(0, row, ptr, k.float().cpu().numpy().astype(np.float64), v.float().cpu().numpy().astype(np.float64))
    ctx.hx_kv_write(pool, 0, seqs, sh.i32(row), sh.i32(ptr), k, v)
    assert status(ctx) == 0
    same(model, pool, seqs)


@pytest.mark.parametrize("n", [16, 17, 255, 1024, 1030, 2100])
def test_forks_and_growth_of_many_rows(ctx, n):
    """Around the number of rows that are compared in one place and the one that is planned at once; some rows are listed twice."""
    rng = np.random.default_rng(n)
    T, parents = 8, 20
    lens = rng.integers(0, 5 * T, parents).tolist()
    model, pool, seqs = make_cache(18, lens, T, layers=1, heads=1, dim=16, rows=parents + n, max_pages=12, spare=6 * n)
    src, dst = rng.integers(0, parents, n), parents + rng.permutation(n)
    twice = rng.permutation(n)[:8]
    dst[twice[:4]] = dst[twice[4:]]
    assert model.fork(src, dst) == {-6}
    ctx.hx_kv_fork(pool, seqs, sh.i32(src), sh.i32(dst))
    assert status(ctx) == -6
    same(model, pool, seqs)
    row, new = rng.permutation(parents + n)[:n], rng.integers(0, 2 * T, n)
    row[twice[:4]] = row[twice[4:]]
    assert model.grow(row, new) == {-6}
    ctx.hx_kv_grow(pool, seqs, sh.i32(row), sh.i32(new))
    assert status(ctx) == -6
    same(model, pool, seqs, numbers=False)


def test_keep_refuses_numbers_out_of_order_and_shared_pages(ctx):
    model, pool, seqs = make_cache(10, [24, 30, 40, 12], 8, rows=8)
    model.fork([2], [5])
    ctx.hx_kv_fork(pool, seqs, sh.i32([2]), sh.i32([5]))
    row, drafts = [0, 0, 1, 1, 2, 3], [9, 9, 4, 4, 10, 13]
    kept = [[2, 5], [1], [3, 1], [4], [4], [0]]
    #   carried out; listed again; falling; too large a number (and listed again); a page that row 5 holds too; more drafts than tokens
    ptr = np.concatenate([[0], np.cumsum([len(x) for x in kept])])
    model.keep(row[:1], drafts[:1], kept[:1])
    ctx.hx_kv_keep(pool, seqs, sh.i32(row), sh.i32(drafts), sh.i32(ptr), sh.i32(sum(kept, [])))
    assert status(ctx) == -6
    same(model, pool, seqs)


def test_free_whole_rows_and_what_a_window_left(ctx):
    model, pool, seqs = make_cache(11, [40, 41, 7, 0, 64], 8, rows=9)
    model.fork([0, 1], [6, 7])
    ctx.hx_kv_fork(pool, seqs, sh.i32([0, 1]), sh.i32([6, 7]))
    row, first, last = [0, 1, 4, 2, 6], [4, 8, -5, 0, 0], [30, 16, 1000, 7, 2]
    model.give(row, first, last)
    ctx.hx_kv_free(pool, seqs, sh.i32(row), sh.i32(first), sh.i32(last))
    assert status(ctx) == 0
    same(model, pool, seqs)
    model.give([0, 7, 3])
    ctx.hx_kv_free(pool, seqs, sh.i32([0, 7, 3, 0]))      # a row listed twice gives back once
    assert status(ctx) == 0
    same(model, pool, seqs)
    ctx.hx_kv_free(pool, seqs, sh.i32([1, 99, -1]))
    model.give([1])
    assert status(ctx) == -6
    same(model, pool, seqs)


def test_free_of_what_lies_beyond_a_row(ctx):
    """Pages of one token, and bounds up to the ends of an int: what they leave out stays."""
    low, high = -2 ** 31, 2 ** 31 - 1
    lens = [40, 0, 7, 300, 1]
    for T in (1, 8):
        model, pool, seqs = make_cache(21, lens, T, rows=9)
        row = [0, 1, 2, 3, 4, 0, 2, 3, 3, 2]
        first = [high, high, high - 255, 300, 1, low, 7, 257, high - 256, low]
        last = [high, 0, high, high, low, low, high, high, low, 3]
        model.give(row, first, last)
        ctx.hx_kv_free(pool, seqs, sh.i32(row), sh.i32(first), sh.i32(last))
        assert status(ctx) == 0
        same(model, pool, seqs)


@pytest.mark.parametrize("n,spare,T", [(0, 5, 8), (3, 0, 8), (12, 40, 4), (200, 900, 1), (3000, 20000, 1)])
def test_compact_moves_pages_down(ctx, n, spare, T):
    rng = np.random.default_rng(n)
    lens = rng.integers(0, 4 * T, n).tolist()
    model, pool, seqs = make_cache(12, lens, T, layers=2, heads=1, dim=16, rows=n + 2, spare=spare)
    import torch
    n_used, moved = torch.full((1,), -7, dtype=torch.int32, device="cuda:0"), torch.full((len(model.ref),), -7, dtype=torch.int32, device="cuda:0")
    want, where = model.compact()
    ctx.hx_kv_compact(pool, seqs, n_used=n_used, moved=moved)
    assert status(ctx) == 0
    assert int(n_used) == want and np.array_equal(moved.cpu().numpy(), where)
    same(model, pool, seqs)
    ctx.hx_kv_compact(pool, seqs)
    assert status(ctx) == 0
    same(model, pool, seqs)


def test_keep_of_bounds_that_are_none(ctx):
    """Ends of a row's list that lie before its start, by so much that their difference passes 32 bits."""
    model, pool, seqs = make_cache(13, [24, 30], 8)
    for ptr in ([2147483647, -2147483647, -2147483647], [2, 0, 1], [-5, 1, 1], [0, 2147483647, -2147483648], [-2147483648, 2147483647, 3]):
        ctx.hx_kv_keep(pool, seqs, sh.i32([0, 1]), sh.i32([0, 0]), sh.i32(ptr), sh.i32([0, 1, 2]))
        assert status(ctx) == -6
    same(model, pool, seqs)


def test_counts_below_none_are_free_pages(ctx):
    model, pool, seqs = make_cache(14, [24, 30, 5], 8, spare=6)
    low = np.nonzero(model.ref == 0)[0][:3]
    pool["ref"][sh.i32(low).long()] = -7
    model.compact()
    ctx.hx_kv_compact(pool, seqs)
    assert status(ctx) == 0
    assert np.array_equal(seqs["table"].cpu().numpy(), model.table) and np.array_equal(np.maximum(pool["ref"].cpu().numpy(), 0), model.ref)


def test_a_row_of_as_many_entries_as_an_int_counts(ctx):
    """Pages of one token, and a row's last ones: taken, filled, dropped again, given back, moved."""
    import torch
    n, new = 2 ** 31 - 1, 300
    table = torch.full((1, n), -1, dtype=torch.int32, device="cuda:0")
    seqs = dict(table=table, len=sh.i32([n - new]))
    k, v = (torch.zeros(1, 2 * new, 1, 1, 16, dtype=torch.bfloat16, device="cuda:0") for _ in range(2))
    pool = dict(k=k, v=v, ref=sh.i32([1, 0] * new))               # every second page is someone else's
    x = torch.arange(new, device="cuda:0").remainder(200).to(torch.bfloat16)[:, None, None].expand(new, 1, 16).contiguous()

    def end():
        assert status(ctx) == 0
        assert bool((table[0, :n - new] == -1).all())
        return table[0, n - new:].tolist(), pool["ref"].tolist(), int(seqs["len"])
    ctx.hx_kv_grow(pool, seqs, sh.i32([0]), sh.i32([new]))
    assert end() == (list(range(1, 2 * new, 2)), [1, 1] * new, n)
    ctx.hx_kv_write(pool, 0, seqs, sh.i32([0]), sh.i32([0, new]), x, -x)
    ctx.hx_kv_keep(pool, seqs, sh.i32([0]), sh.i32([new]), sh.i32([0, 3]), sh.i32([0, 7, 299]))
    assert end() == ([1, 3, 5] + [-1] * (new - 3), [1, 1] * 3 + [1, 0] * (new - 3), n - new + 3)
    assert [k[0, p, 0, 0, 5].item() for p in (1, 3, 5)] == [0, 7, 99] and torch.equal(k, -v)
    ctx.hx_kv_grow(pool, seqs, sh.i32([0]), sh.i32([new - 3]))
    ctx.hx_kv_free(pool, seqs, sh.i32([0, 0, 0]), sh.i32([n - 260, n, n]), sh.i32([n, n, 2 ** 31 - 1]))
    assert end() == (list(range(1, 81, 2)) + [-1] * 260, [1, 1] * 40 + [1, 0] * 260, n)
    ctx.hx_kv_compact(pool, seqs)
    got, ref, _ = end()
    assert ref == [1] * 340 + [0] * 260 and got[:40] == list(range(1, 81, 2)) and got[40:] == [-1] * 260


def test_fork_of_entries_that_are_no_pages(ctx):
    model, pool, seqs = make_cache(15, [30, 16], 8, rows=6)
    seqs["table"][0, 1] = seqs["table"][0, 3] = len(model.ref)
    ctx.hx_kv_fork(pool, seqs, sh.i32([0, 1]), sh.i32([4, 5]))
    assert status(ctx) == -6
    model.table[0, 1] = model.table[0, 3] = -1
    model.fork([0, 1], [4, 5])
    model.table[0, 1] = model.table[0, 3] = len(model.ref)
    same(model, pool, seqs)


# ---- attention -----------------------------------------------------------------------------------------------------------

def check_attend(ctx, lens, nq, heads=2, group=2, dim=64, T=16, type_="bf16", cache=None, window=0, sinks=0, parents=None, scale=None,
                 missing=(), q_layout="wide", max_len=None, seed=0, layers=2, layer=1, garbage=True, peaks=0.0, skip=()):
    """One call over a cache of these lengths (the last nq[i] tokens query) against the plain form; `missing`: (sequence, block) without a
    page; `skip`: sequences whose outputs are not compared."""
    import torch
    cache = cache or type_
    rng = np.random.default_rng(seed)
    g = torch.Generator().manual_seed(seed)
    n, hq = len(lens), heads * group
    need = [-(-x // T) for x in lens]
    n_pages = sum(need) + 5
    order = rng.permutation(n_pages)
    rows = n + 3
    where = rng.permutation(rows)[:n]                       # sequence i lies in row where[i]
    table, at = np.full((rows, max(need + [1]) + 1), -1), 0
    for i in range(n):
        table[where[i], :need[i]] = order[at:at + need[i]]
        at += need[i]
    shape = (layers, n_pages, heads, T, dim)
    full = torch.randn((2,) + shape, generator=g)
    if peaks:
        full[0] *= peaks
    k_scale = v_scale = None
    if cache == "e4m3":
        full *= 30
        k_scale, v_scale = (torch.rand(layers, heads, generator=g) + 0.5) / 30, (torch.rand(layers, heads, generator=g) + 0.5) / 30
    full = full.to(sh.torch_type(cache))
    kk, vv = (x.float().numpy().astype(np.float64) for x in full)
    if k_scale is not None:
        kk, vv = kk * k_scale.double().numpy()[:, None, :, None, None], vv * v_scale.double().numpy()[:, None, :, None, None]
    if garbage:
        # what no sequence may see: pages of nobody, and what lies behind a sequence's end in its last page
        bad = torch.full((dim,), float("nan")).to(sh.torch_type(cache))
        for p in order[at:]:
            full[:, :, p] = bad
        for i in range(n):
            if lens[i] % T:
                full[:, :, table[where[i], need[i] - 1], :, lens[i] % T:] = bad
    length = np.zeros(rows, np.int64)
    length[where] = lens
    for i, b in missing:
        if garbage:
            full[:, :, table[where[i], b]] = float("nan")
        table[where[i], b] = -1
    pool = dict(k=full[0].cuda().contiguous(), v=full[1].cuda().contiguous(), ref=sh.i32(np.ones(n_pages)), page_tokens=T)
    if k_scale is not None:
        pool["k_scale"], pool["v_scale"] = k_scale.cuda(), v_scale.cuda()
    ptr = np.concatenate([[0], np.cumsum(nq)])
    total = int(ptr[-1])
    t = sh.torch_type(type_)
    if q_layout == "wide":
        q = torch.randn(total, hq + 2, dim, generator=g).to(t).cuda()[:, 1:-1]
        out = torch.full((total, hq, dim), 7.0, dtype=t, device="cuda:0")
    else:                                                    # heads before tokens, nothing aligned
        q = torch.randn(hq, total, dim + 1, generator=g).to(t).cuda()[:, :, 1:].transpose(0, 1)
        out = torch.full((hq, total, dim + 1), 7.0, dtype=t, device="cuda:0")[:, :, 1:].transpose(0, 1)
    lse = torch.full((total, hq), 7.0, device="cuda:0")
    par = None if parents is None else sh.i32(np.concatenate([np.asarray(p, np.int64) for p in parents] + [np.zeros(0, np.int64)]))
    ctx.hx_attend(pool, layer, dict(table=sh.i32(table), len=sh.i32(length)), sh.i32(ptr), q, out, max_q=max(list(nq) + [1]), max_len=max_len,
                  row=sh.i32(where), scale=scale, window=window, n_sink=sinks, parent=par, lse=lse)
    code = status(ctx)
    got, got_lse = out.float().cpu().numpy().astype(np.float64), lse.cpu().numpy().astype(np.float64)
    qf = q.float().cpu().numpy().astype(np.float64)
    step, scale = sh.HALF_STEP[type_], dim ** -0.5 if scale is None else scale
    for i in range(n):
        if i in skip or nq[i] == 0:
            continue
        see = sh.visible(lens[i], nq[i], None if parents is None else parents[i], window, sinks)
        for j, b in missing:
            if j == i:
                see[:, b * T:(b + 1) * T] = False
        pages = np.maximum(table[where[i], :need[i]], 0)
        k, v = (x[layer, pages].transpose(0, 2, 1, 3).reshape(-1, heads, dim)[:lens[i]] for x in (kk, vv))
        o, l, size, plain, reach = sh.attend(qf[ptr[i]:ptr[i + 1]], k, v, see, scale, group)
        mine, mine_lse = got[ptr[i]:ptr[i + 1]], got_lse[ptr[i]:ptr[i + 1]]
        # scores: dim products and as many sums in 32 bits; the exponent's argument a few more roundings; sums of weights in 32 bits
        ds = (dim + 8) * 2.0 ** -24 * reach + 2.0 ** -21
        sums = (see.sum(1)[:, None] + 16) * 2.0 ** -24
        near = (step + 2 * ds + sums)[..., None] * size + step * np.abs(o) + 1e-30
        if type_ == "f16":
            near = near + 2.0 ** -25 * plain + 2.0 ** -25     # weights and outputs below the least normal number
        assert np.array_equal(np.isinf(l), np.isinf(mine_lse)) and (mine_lse[np.isinf(l)] < 0).all()
        fin = np.isfinite(l)
        assert (np.abs(mine_lse - l)[fin] <= (ds + sums + 2.0 ** -22 * np.abs(np.where(fin, l, 0)))[fin]).all()
        assert (mine[~fin] == 0).all()
        far = np.abs(mine - o) - near
        assert (far <= 0).all(), (i, np.unravel_index(far.argmax(), far.shape), far.max(), np.abs(mine - o).max())
    return code, got, got_lse


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("type_,cache", [("bf16", "bf16"), ("f16", "f16"), ("bf16", "e4m3"), ("f16", "e4m3")])
def test_one_query_each(ctx, dim, type_, cache):
    lens = [1, 2, 15, 16, 17, 63, 64, 65, 130, 257, 700]
    assert check_attend(ctx, lens, [1] * len(lens), dim=dim, type_=type_, cache=cache)[0] == 0


@pytest.mark.parametrize("heads,group", [(1, 1), (1, 7), (3, 1), (2, 3), (1, 16), (1, 17), (2, 33), (8, 4)])
def test_head_layouts(ctx, heads, group):
    assert check_attend(ctx, [5, 90, 200], [1, 3, 2], heads=heads, group=group)[0] == 0


@pytest.mark.parametrize("T", [1, 2, 8, 16, 32, 64, 256, 1024])
def test_page_sizes(ctx, T):
    assert check_attend(ctx, [3, 100, 333], [1, 5, 40], T=T, window=70, sinks=3)[0] == 0


@pytest.mark.parametrize("window", [0, 1, 2, 17, 64, 65, 500])
@pytest.mark.parametrize("sinks", [0, 1, 5, 64, 70, 1000])
def test_windows_and_sinks(ctx, window, sinks):
    lens = [1, 40, 64, 129, 300, 411]
    assert check_attend(ctx, lens, [1] * 6, window=window, sinks=sinks)[0] == 0
    assert check_attend(ctx, lens, [1, 40, 9, 70, 150, 33], group=3, heads=1, window=window, sinks=sinks, seed=1)[0] == 0


@pytest.mark.parametrize("dim,type_,cache", [(64, "bf16", "bf16"), (128, "f16", "f16"), (128, "bf16", "e4m3"), (256, "bf16", "bf16"), (256, "f16", "e4m3")])
@pytest.mark.parametrize("rows", [20, 50, 300])
def test_prompts(ctx, dim, type_, cache, rows):
    lens = [rows, rows + 1, 2 * rows + 77]
    assert check_attend(ctx, lens, [rows, rows - 3, rows], dim=dim, type_=type_, cache=cache, heads=1, group=2)[0] == 0


@pytest.mark.parametrize("rows", [1, 9, 40])
def test_long_contexts_are_divided_and_joined(ctx, rows):
    lens = [4096, 3001]
    for window in (0, 1500):
        assert check_attend(ctx, lens, [rows, 1], heads=1, group=4, dim=128, window=window, sinks=4)[0] == 0


@pytest.mark.parametrize("nq", [[1] * 16, [33, 2, 1, 1, 7, 1, 1, 1]])
def test_few_long_parts_where_the_rows_fill_the_chip(ctx, nq):
    """1024 and 512 tiles of rows: parts of 64 tiles of keys and more, or 128, the last one longer; lengths around their ends."""
    lens = ([6500, 4200, 2500, 1, 700, 64, 2049, 4097] * 2)[:len(nq)]
    for window in (0, 4500):
        assert check_attend(ctx, lens, nq, heads=64, group=1, window=window, sinks=3, layers=1, layer=0)[0] == 0


def tree(rng, n, near, dead=0):
    p = [int(rng.integers(max(-1, i - near), i)) for i in range(n)]
    for i in rng.permutation(n)[:dead]:
        p[i] = -2
    return p


@pytest.mark.parametrize("n", [1, 2, 8, 25, 64, 200, 256])
@pytest.mark.parametrize("window,sinks", [(0, 0), (3, 0), (20, 2), (400, 9)])
def test_trees(ctx, n, window, sinks):
    rng = np.random.default_rng(n)
    lens = [n, n + 1, n + 100, n + 333]
    parents = [tree(rng, n, near) for near in (1, 4, 300, 9)]
    assert check_attend(ctx, lens, [n] * 4, heads=1, group=3, dim=128, window=window, sinks=sinks, parents=parents)[0] == 0


def test_trees_with_drafts_left_out(ctx):
    rng = np.random.default_rng(0)
    parents = [tree(rng, 30, 5, 8), [-2] * 12, [-2, 0, 1, -1], [-1]]
    code, out, lse = check_attend(ctx, [150, 12, 60, 1], [30, 12, 4, 1], parents=parents)
    assert code == 0
    assert (out[30:45] == 0).all() and np.isinf(lse[30:45]).all()


def test_trees_with_parents_out_of_range(ctx):
    parents = [[-1, 0, 2, 0, 9], [-1, -7, 1, 0, 0], [-1] * 4]
    read = [[-1, 0, -2, 0, -2], [-1, -2, 1, 0, 0], [-1] * 4]
    assert check_attend(ctx, [50, 60, 40], [5, 5, 4], parents=parents, skip=(0, 1))[0] == -6
    code, out, lse = check_attend(ctx, [50, 60, 40], [5, 5, 4], parents=parents, skip=(0, 1))
    clean = check_attend(ctx, [50, 60, 40], [5, 5, 4], parents=read)
    assert clean[0] == 0 and np.array_equal(clean[1], out) and np.array_equal(clean[2], lse)


def test_pages_that_are_not_there(ctx):
    missing = [(0, 0), (0, 3), (1, 0), (1, 1), (2, 5), (3, 0)]
    code, out, lse = check_attend(ctx, [100, 30, 96, 1], [1, 2, 50, 1], missing=missing)
    assert code == 0
    assert (out[1:3] == 0).all() and np.isinf(lse[1:3]).all() and (out[-1] == 0).all()


@pytest.mark.parametrize("T", [8, 64])
def test_a_window_reads_the_same_after_its_pages_went(ctx, T):
    lens, window, sinks = [500, 300, 90], 64, 4
    missing = [(i, b) for i, n in enumerate(lens) for b in range(n // T) if b * T >= sinks and (b + 1) * T <= n - window]
    with_all = check_attend(ctx, lens, [1] * 3, T=T, window=window, sinks=sinks)
    without = check_attend(ctx, lens, [1] * 3, T=T, window=window, sinks=sinks, missing=missing)
    assert np.array_equal(with_all[1], without[1]) and np.array_equal(with_all[2], without[2])


@pytest.mark.parametrize("nq", [[1, 1, 1], [3, 70, 20]])
def test_strides_and_alignment(ctx, nq):
    for type_ in ("bf16", "f16"):
        assert check_attend(ctx, [50, 200, 77], nq, q_layout="odd", type_=type_, dim=128)[0] == 0


@pytest.mark.parametrize("scale", [0.0, -0.3, 3.0])
def test_scales(ctx, scale):
    assert check_attend(ctx, [50, 200, 77], [3, 70, 1], scale=scale, window=60, sinks=1)[0] == 0


def test_scores_far_apart(ctx):
    """Maxima that keep moving, and weights that vanish."""
    for type_ in ("bf16", "f16"):
        assert check_attend(ctx, [700, 900], [1, 60], peaks=12.0, type_=type_, dim=128)[0] == 0


@pytest.mark.parametrize("type_,cache", [("f16", "f16"), ("bf16", "bf16"), ("f16", "e4m3")])
@pytest.mark.parametrize("n,nq,group,far", [(32768, 1, 1, 25.2), (32768, 1, 4, 26.9), (20000, 3, 2, 22.0), (6000, 20, 4, 24.9), (3000, 40, 1, 25.5), (700, 1, 2, 28.0)])
def test_many_small_weights_beside_a_large_one(ctx, type_, cache, n, nq, group, far):
    """One key's weight is 2^far of the others', whose values alone are not 0: together they are the result."""
    import torch
    T, dim = 32, 64
    t, step = sh.torch_type(type_), sh.HALF_STEP[type_]
    pages = -(-n // T)
    g = torch.Generator().manual_seed(n)
    k = torch.zeros(1, pages, 1, T, dim)
    k[0, (n - nq) // 2 // T, 0, (n - nq) // 2 % T, 0] = 12.0
    v = 1 + torch.rand(1, pages, 1, T, dim, generator=g)
    v[0, (n - nq) // 2 // T, 0, (n - nq) // 2 % T] = 0
    k, v = k.to(sh.torch_type(cache)).cuda(), v.to(sh.torch_type(cache)).cuda()
    q = torch.zeros(nq, group, dim)
    q[:, :, 0] = far * math.log(2) * dim ** 0.5 / 12.0
    q = q.to(t).cuda()
    out, lse = attend_out(ctx, k, v, sh.i32(np.arange(pages)[None]), sh.i32([n]), sh.i32([0, nq]), q, T)
    kf, vf = (x[0, :, 0].float().reshape(-1, 1, dim)[:n].cpu().numpy().astype(np.float64) for x in (k, v))
    o, l, size, plain, reach = sh.attend(q.double().cpu().numpy(), kf, vf, sh.visible(n, nq, None, 0, 0), dim ** -0.5, group)
    ds = (dim + 8) * 2.0 ** -24 * reach + 2.0 ** -21
    sums = (n + 16) * 2.0 ** -24
    near = (step + 2 * ds[..., None] + sums) * size + step * np.abs(o)
    if type_ == "f16":
        near = near + 2.0 ** -32 * plain + 2.0 ** -25     # weights below the least normal number, 2^7 up; outputs below it
    assert (np.abs(out - o) <= near).all(), (np.abs(out - o) / near).max()
    assert (np.abs(lse - l) <= ds + sums + 2.0 ** -22 * np.abs(l)).all()
    assert status(ctx) == 0


@pytest.mark.parametrize("type_,cache", [("bf16", "bf16"), ("f16", "f16"), ("bf16", "e4m3"), ("f16", "e4m3")])
@pytest.mark.parametrize("dim,nq,group", [(64, 1, 4), (128, 3, 8), (128, 1, 1), (256, 8, 2)])
@pytest.mark.parametrize("n", [90, 5000])
def test_few_rows_are_off_by_their_own_rounding(ctx, type_, cache, dim, nq, group, n):
    """Up to 32 rows a KV head: weights as two numbers, so that hardly more than the rounding of the result remains."""
    import torch
    T, heads = 16, 2
    g = torch.Generator().manual_seed(n + dim)
    pages = -(-n // T)
    k, v = (torch.randn(1, pages, heads, T, dim, generator=g).to(sh.torch_type(cache)).cuda() for _ in range(2))
    q = torch.randn(nq, heads * group, dim, generator=g).to(sh.torch_type(type_)).cuda()
    out, _ = attend_out(ctx, k, v, sh.i32(np.arange(pages)[None]), sh.i32([n]), sh.i32([0, nq]), q, T)
    kf, vf = (x[0].float().cpu().numpy().transpose(0, 2, 1, 3).reshape(-1, heads, dim)[:n].astype(np.float64) for x in (k, v))
    o, _, size, plain, reach = sh.attend(q.double().cpu().numpy(), kf, vf, sh.visible(n, nq, None, 0, 0), dim ** -0.5, group)
    bits = 8 if type_ == "bf16" else 11
    ds = (dim + 8) * 2.0 ** -24 * reach + 2.0 ** -21
    near = (2.0 ** (-2 * bits) + 2 * ds + (n + 16) * 2.0 ** -24)[..., None] * size
    if type_ == "f16":
        near = near + 2.0 ** -32 * plain + 2.0 ** -25
    # half a step of the result, or of the one above where the sums take it there
    near = near + 2.0 ** (np.floor(np.log2(np.abs(o) + near)) - bits)
    assert (np.abs(out - o) <= near).all(), (np.abs(out - o) / near).max()
    assert status(ctx) == 0


def test_how_the_work_is_divided_does_not_go_by_the_real_lengths(ctx):
    for most in (0, 1, 100, 100000):
        assert check_attend(ctx, [700, 30, 4000], [1, 2, 5], max_len=most, heads=1, dim=128)[0] == 0


def test_rows_and_queries_out_of_range(ctx):
    import torch
    from paper_2605_16637_amd import binding
    x = torch.zeros(1, 8, 1, 16, 64, dtype=torch.bfloat16, device="cuda:0")
    pool = dict(k=x, v=torch.ones_like(x), ref=sh.i32(np.ones(8)))
    seqs = dict(table=sh.i32([[0, 1], [2, 9], [3, 4]]), len=sh.i32([20, 20, 33]))
    q = torch.zeros(4, 1, 64, dtype=torch.bfloat16, device="cuda:0")

    def call(row, ptr, max_q=2):
        out, lse = torch.full_like(q, 7.0), torch.full((4, 1), 7.0, device="cuda:0")
        ctx.hx_attend(pool, 0, seqs, sh.i32(ptr), q, out, max_q=max_q, row=sh.i32(row), lse=lse)
        code = status(ctx)
        return code, out.float().cpu().numpy()[:, 0], lse.cpu().numpy()[:, 0]
    code, out, lse = call([0, 5, -1], [0, 1, 2, 3])
    assert code == -6 and (out[0] == 1).all() and (out[1:3] == 0).all() and np.isneginf(lse[1:3]).all() and (out[3] == 7).all()
    code, out, _ = call([1, 2, 0], [0, 1, 2, 3])             # a page out of range is not there; a length beyond the table
    assert code == -6 and (out[0] == 1).all() and (out[1] == 0).all() and (out[2] == 1).all()
    assert call([0], [0, 9])[0] == -6
    assert call([0, 0], [0, 3, 1])[0] == -6
    code, out, _ = call([0], [0, 4], max_q=2)                # more queries than max_q says
    assert code == -6
    with pytest.raises(binding.HxError):
        call([0], [0, 300], max_q=-1)


def test_nothing_to_do(ctx):
    import torch
    assert check_attend(ctx, [0, 0], [0, 0])[0] == 0
    assert check_attend(ctx, [0, 5, 40], [0, 0, 2])[0] == 0
    x = torch.zeros(1, 0, 1, 16, 64, dtype=torch.bfloat16, device="cuda:0")
    ctx.hx_kv_compact(dict(k=x, v=x, ref=sh.i32([])), dict(table=sh.i32(np.zeros((0, 0))), len=sh.i32([])))
    assert status(ctx) == 0


def attend_out(ctx, k, v, table, length, ptr, q, T, **more):
    """(out, lse) in 64 bits of one call over layer 0 of a bf16 or fp16 cache."""
    import torch
    out, lse = torch.full_like(q, 7.0), torch.full(q.shape[:2], 7.0, device="cuda:0")
    ctx.hx_attend(dict(k=k, v=v, ref=sh.i32(np.ones(k.shape[1]))), 0, dict(table=table, len=length), ptr, q, out, max_q=int(ptr.diff().max()), lse=lse, **more)
    return out.float().cpu().numpy().astype(np.float64), lse.cpu().numpy().astype(np.float64)


@pytest.mark.parametrize("type_", ["bf16", "f16"])
@pytest.mark.parametrize("dim,group,nq,T,is_tree", [(64, 1, 9, 16, False), (64, 4, 60, 16, False), (128, 2, 16, 8, False), (128, 4, 70, 32, False), (128, 3, 5, 16, True),
                                                    (128, 4, 40, 16, True), (256, 2, 14, 16, True), (256, 4, 33, 4, False), (64, 2, 300, 16, False)])
def test_infinite_and_nan_values_that_some_queries_do_not_see(ctx, type_, dim, group, nq, T, is_tree):
    """Keys and values of some positions are replaced; rows that do not see these keep their results, the others' follow the formula."""
    import torch
    n = nq + 700
    rng = np.random.default_rng(nq)
    g = torch.Generator().manual_seed(nq)
    t = sh.torch_type(type_)
    pages = -(-n // T)
    k, v = (torch.randn(1, pages, 1, T, dim, generator=g).to(t).cuda() for _ in range(2))
    q = torch.randn(nq, group, dim, generator=g).to(t).cuda()
    table, length, ptr = sh.i32(rng.permutation(pages)[None]), sh.i32([n]), sh.i32([0, nq])
    parent = tree(rng, nq, 5, 2) if is_tree else None
    window, sinks = 600, 3
    more = dict(window=window, n_sink=sinks, parent=None if parent is None else sh.i32(parent))
    see = sh.visible(n, nq, parent, window, sinks)
    was, was_lse = attend_out(ctx, k, v, table, length, ptr, q, T, **more)
    # each within (half a step of the weights + of the output, and sums in 32 bits) of the exact result, at most the largest |value|
    near = 2 * (2 * sh.HALF_STEP[type_] + 2.0 ** -12) * float(v.float().abs().max())
    place = table[0].cpu().numpy()
    seen_by_some = np.nonzero(see.any(0) & ~see[see.any(1)].all(0))[0]
    assert len(seen_by_some)
    unseen = np.nonzero(~see.any(0))[0][-1:].tolist()
    odd = sorted(set([int(seen_by_some[0]), int(seen_by_some[len(seen_by_some) // 4]), int(seen_by_some[-1])] + [int(x) for x in unseen]))
    for what in (float("inf"), float("-inf"), float("nan")):
        v2 = v.clone()
        for y in odd:
            v2[0, place[y // T], 0, y % T, 1::3] = what
        got, lse = attend_out(ctx, k, v2, table, length, ptr, q, T, **more)
        hit = see[:, odd].any(1)
        assert (~hit).any() or is_tree
        assert np.array_equal(lse, was_lse)
        assert (np.abs(got - was)[~hit] <= near).all()
        plain = np.ones(dim, bool)
        plain[1::3] = False
        assert (np.abs(got - was)[hit][..., plain] <= near).all()
        x = got[hit][..., ~plain]
        assert np.isnan(x).all() if what != what else (x == what).all()
    k2 = k.clone()
    for y in odd:
        k2[0, place[y // T], 0, y % T] = float("nan")
        v2[0, place[y // T], 0, y % T] = float("nan")
    got, lse = attend_out(ctx, k2, v2, table, length, ptr, q, T, **more)
    assert np.isnan(got[hit]).all() and np.isnan(lse[hit]).all()
    # (how far a maximum has been raised goes by the rows beside it: sums of n weights in 32 bits, twice)
    sums = 2 * (n + 64) * 2.0 ** -24 * np.maximum(1.0, np.abs(was_lse[~hit], where=np.isfinite(was_lse[~hit]), out=np.zeros_like(was_lse[~hit])))
    near_lse = (lse[~hit] == was_lse[~hit]) | (np.abs(np.where(np.isfinite(lse[~hit]), lse[~hit], 0) - np.where(np.isfinite(was_lse[~hit]), was_lse[~hit], 0)) <= sums)
    assert (np.abs(got - was)[~hit] <= near).all() and near_lse.all() and np.array_equal(np.isinf(lse[~hit]), np.isinf(was_lse[~hit]))
    assert status(ctx) == 0


@pytest.mark.parametrize("type_,cache", [("bf16", "bf16"), ("f16", "f16")])
@pytest.mark.parametrize("dim,group,n", [(64, 1, 5), (128, 4, 3000), (128, 20, 700), (256, 2, 90), (64, 40, 700), (128, 40, 6000)])
def test_a_single_token_that_sees_infinite_values(ctx, type_, cache, dim, group, n):
    """Weights are above 0: an infinite value leaves its sum infinite, two of opposite signs leave none, and other numbers stay as they are."""
    import torch
    T = 16
    g = torch.Generator().manual_seed(n)
    k, v = (torch.randn(1, -(-n // T), 1, T, dim, generator=g).to(sh.torch_type(cache)).cuda() for _ in range(2))
    q = torch.randn(1, group, dim, generator=g).to(sh.torch_type(type_)).cuda()
    args = (sh.i32(np.arange(-(-n // T))[None]), sh.i32([n]), sh.i32([0, 1]), q, T)
    was, was_lse = attend_out(ctx, k, v, *args)
    at = [1, n // 2, n - 1]
    for y in at:
        v[0, y // T, 0, y % T, 1] = float("inf")
        v[0, y // T, 0, y % T, 2] = float("-inf")
        v[0, y // T, 0, y % T, 3] = float("inf") if y == at[0] else float("-inf")
    got, lse = attend_out(ctx, k, v, *args)
    assert (got[..., 1] == np.inf).all() and (got[..., 2] == -np.inf).all() and np.isnan(got[..., 3]).all()
    assert np.array_equal(lse, was_lse)
    rest = np.arange(dim) > 3
    near = 2 * (2 * sh.HALF_STEP[type_] + 2.0 ** -12) * float(v.float().abs()[..., 4:].max())
    assert (np.abs(got - was)[..., rest] <= near).all()
    assert status(ctx) == 0


def test_a_single_token_that_sees_no_number(ctx):
    import torch
    g = torch.Generator().manual_seed(1)
    for n in (5, 3000):
        k, v = (torch.randn(1, -(-n // 16), 2, 16, 64, generator=g).to(torch.bfloat16).cuda() for _ in range(2))
        q = torch.randn(1, 4, 64, generator=g).to(torch.bfloat16).cuda()
        k[0, 0, 1, 2] = float("nan")
        got, lse = attend_out(ctx, k, v, sh.i32(np.arange(-(-n // 16))[None]), sh.i32([n]), sh.i32([0, 1]), q, 16)
        assert np.isfinite(got[0, :2]).all() and np.isfinite(lse[0, :2]).all() and np.isnan(got[0, 2:]).all() and np.isnan(lse[0, 2:]).all()


@pytest.mark.parametrize("type_", ["bf16", "f16"])
@pytest.mark.parametrize("dim,group,T,context,window,sinks,others", [
    (64, 1, 16, 700, 100, 0, []), (64, 4, 16, 700, 96, 4, []), (128, 4, 8, 300, 33, 3, [5, 2]), (128, 3, 32, 6000, 5000, 1, []),
    (64, 40, 16, 700, 100, 0, []), (128, 48, 8, 333, 64, 7, []), (128, 4, 16, 500, 64, 2, [40, 12]), (256, 4, 16, 90, 1, 0, []), (256, 33, 4, 90, 17, 2, [3])])
def test_a_tree_of_one_draft_does_not_see_what_lies_before_its_window(ctx, type_, dim, group, T, context, window, sinks, others):
    """One draft, alone and beside larger trees; the values of the last position before the window, and of all that no window holds, are replaced."""
    import torch
    nq = [1] + others
    lens = [context + m for m in nq]
    g = torch.Generator().manual_seed(context)
    t = sh.torch_type(type_)
    per = [-(-n // T) for n in lens]
    table = np.full((len(lens), max(per)), -1)
    at = 0
    for i, k in enumerate(per):
        table[i, :k] = np.arange(at, at + k)
        at += k
    k, v = (torch.randn(1, at, 1, T, dim, generator=g).to(t).cuda() for _ in range(2))
    q = torch.randn(sum(nq), group, dim, generator=g).to(t).cuda()
    parent = sh.i32(np.concatenate([np.arange(-1, m - 1) for m in nq]))
    more = dict(window=window, n_sink=sinks, parent=parent)
    args = (sh.i32(table), sh.i32(lens), sh.i32(np.concatenate([[0], np.cumsum(nq)])), q, T)
    was, was_lse = attend_out(ctx, k, v, *args, **more)
    see = sh.visible(lens[0], 1, [-1], window, sinks)[0]
    assert not see[context - window] and see[context - window + 1:].all()
    for what in (float("inf"), float("-inf"), float("nan")):
        for which in ([context - window], np.nonzero(~see)[0]):
            k2, v2 = k.clone(), v.clone()
            for y in which:
                v2[0, table[0, y // T], 0, y % T] = what
                if what != what:
                    k2[0, table[0, y // T], 0, y % T] = what
            got, lse = attend_out(ctx, k2, v2, *args, **more)
            assert np.isfinite(got).all() and np.array_equal(got, was) and np.array_equal(lse, was_lse), (what, len(which))
        v2[0, table[0, (context - window + 1) // T], 0, (context - window + 1) % T, 5] = what        # the first that it sees
        got, _ = attend_out(ctx, k, v2, *args, **more)
        assert not np.isfinite(got[0, :, 5]).any() and np.isfinite(got[0][:, np.arange(dim) != 5]).all()
    assert status(ctx) == 0


@pytest.mark.parametrize("type_,cache,dim", [("bf16", "bf16", 256), ("f16", "e4m3", 128), ("bf16", "e4m3", 64)])
@pytest.mark.parametrize("nq", [1, 30])
def test_the_first_call_of_a_context_may_be_captured(type_, cache, dim, nq):
    import torch
    from paper_2605_16637_amd import binding
    g = torch.Generator().manual_seed(dim)
    n, T, t = 60, 16, sh.torch_type(type_)
    k, v = (torch.randn(1, 4, 2, T, dim, generator=g).to(sh.torch_type(cache)).cuda() for _ in range(2))
    q = torch.randn(nq, 4, dim, generator=g).to(t).cuda()
    pool, seqs = dict(k=k, v=v, ref=sh.i32(np.ones(4))), dict(table=sh.i32([[2, 0, 3, 1]]), len=sh.i32([n]))
    ptr, parent = sh.i32([0, nq]), sh.i32(np.arange(-1, nq - 1))
    out, want = torch.zeros_like(q), torch.zeros_like(q)
    c, other = binding.Context(0), binding.Context(0)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.hx_attend(pool, 0, seqs, ptr, q, out, max_q=nq, max_len=n, parent=parent)
    other.hx_attend(pool, 0, seqs, ptr, q, want, max_q=nq, max_len=n, parent=parent)
    for _ in range(3):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and bool(want.float().abs().sum() > 0)
    assert status(c) == 0 and status(other) == 0
    c.close()
    other.close()


def test_scratch_does_not_grow_while_a_stream_is_captured():
    import torch
    from paper_2605_16637_amd import binding
    c = binding.Context(0)
    model, pool, seqs = make_cache(31, [9, 4], 8, rows=4)
    begin = [x.clone() for x in (seqs["table"], seqs["len"], pool["ref"])]
    row, one = sh.i32([0, 1]), sh.i32([1, 9])
    graph, x = torch.cuda.CUDAGraph(), torch.zeros(8, device="cuda:0")
    with torch.cuda.graph(graph):
        x += 1
        with pytest.raises(binding.HxError) as e:
            c.hx_kv_grow(pool, seqs, row, one)
    assert e.value.code == -4
    graph.replay()
    torch.cuda.synchronize()
    assert float(x[0]) == 1 and all(torch.equal(a, b) for a, b in zip(begin, (seqs["table"], seqs["len"], pool["ref"])))
    c.hx_kv_grow(pool, seqs, row, one)
    model.grow([0, 1], [1, 9])
    assert status(c) == 0
    same(model, pool, seqs)
    c.close()


# ---- sampling ------------------------------------------------------------------------------------------------------------

def check_sample(ctx, x, u, type_="f32", T=None, k=None, p=None, mp=None, pad=0):
    """One call on logits x (float64 [rows, vocabulary]) against the plain form.  Sums of the plain form are off by n 2^-53 of the whole at most;
    where a limit lies nearer than that the row is not one to test with, and there is none in these tests."""
    import torch
    n, v = x.shape
    t = torch.empty(n, v + pad, dtype=sh.torch_type(type_), device="cuda:0")
    t[:, :v] = torch.as_tensor(x).to(sh.torch_type(type_)).cuda()
    logits = t[:, :v]
    f = lambda y: None if y is None else sh.dev(np.asarray(y, np.float32))  # noqa: E731
    token, kept = (torch.full((n,), -7, dtype=torch.int32, device="cuda:0") for _ in range(2))
    logprob = torch.full((n,), 7.0, device="cuda:0")
    ctx.hx_sample(logits, f(u), token, temperature=f(T), top_k=None if k is None else sh.i32(k), top_p=f(p), min_p=f(mp), logprob=logprob, n_kept=kept)
    code = status(ctx)
    xs = logits.double().cpu().numpy()
    get = lambda y, i, d: d if y is None else float(np.float32(y[i]))  # noqa: E731
    for i in range(n):
        row = np.where(np.isnan(xs[i]), -np.inf, xs[i])
        want = sh.sample(row, get(T, i, 1.0), int(get(k, i, 0)), get(p, i, 1.0), get(mp, i, 0.0), float(np.float32(u[i])))
        assert (int(token[i]), int(kept[i])) == (want[0], want[2]), (i, int(token[i]), int(kept[i]), want)
        got = float(logprob[i])
        assert got == want[1] or abs(got - want[1]) <= 2.0 ** -24 * abs(want[1]) + 1e-9, (i, got, want)
    return code, token.cpu().numpy()


@pytest.mark.parametrize("type_", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("v", [1, 2, 7, 64, 500, 1023, 8192, 32003])
def test_sample_settings(ctx, type_, v):
    rng = np.random.default_rng(v)
    n = 24
    x = rng.normal(0, 2.5, (n, v)) + (rng.random((n, v)) < 0.002) * 6
    x[rng.random((n, v)) < 0.02] = -np.inf
    x[:, rng.integers(0, v)] = 1.0
    T = rng.uniform(0.3, 1.5, n)
    T[3], T[7] = 0.0, 1e-3
    k = np.where(rng.random(n) < 0.5, rng.integers(1, 3 + v // 3, n), 0)
    p = np.where(rng.random(n) < 0.6, rng.uniform(0.05, 0.999, n), 1.0)
    mp = np.where(rng.random(n) < 0.4, rng.uniform(0.001, 0.5, n), 0.0)
    u = rng.random(n)
    for pad in (0, 3):
        assert check_sample(ctx, x, u, type_, T, k, p, mp, pad)[0] == 0
    assert check_sample(ctx, x, u, type_)[0] == 0
    assert check_sample(ctx, x, u, type_, T=T)[0] == 0
    assert check_sample(ctx, x, u, type_, k=k)[0] == 0
    assert check_sample(ctx, x, u, type_, p=p)[0] == 0
    assert check_sample(ctx, x, u, type_, mp=mp)[0] == 0


def test_sample_equal_logits_go_to_the_lowest_numbers(ctx):
    for v in (3, 1000, 20000):
        x = np.zeros((6, v))
        x[1, v // 2:] = 1.0
        x[2, 1::2] = -0.0
        assert check_sample(ctx, x, [0.0, 0.5, 0.999999, 0.25, 0.3, 0.9], "f32", k=[2, 1, 0, v, 3, v - 1])[0] == 0
        assert check_sample(ctx, x, [0.0, 0.5, 0.9999, 0.25, 0.3, 0.7], "bf16", p=[0.5, 0.25, 0.75, 1.0, 0.001, 0.0])[0] == 0
        assert check_sample(ctx, x, [0.0, 0.5, 0.75, 0.25, 0.3, 0.9], "f16", mp=[1.0] * 6)[0] == 0
        assert check_sample(ctx, x, [0.0, 0.5, 0.75, 0.25, 0.3, 0.9], "f32", T=[0.0] * 6)[0] == 0


def test_sample_ends_of_the_range(ctx):
    x = np.full((8, 300), -3.0)
    x[0] = -np.inf                                            # nothing is left
    x[1, :] = -np.inf
    x[1, 77] = -3.4e38
    x[2, :] = -3.4028234663852886e38                          # masked with the type's lowest value, all of it and all but one
    x[3, :] = -3.4028234663852886e38
    x[3, 5] = 2.0
    x[4, [9, 200]] = np.inf
    x[5, 0], x[5, 1:] = 3.4e38, -3.4e38
    x[6, ::2] = 1e-42
    x[7, 3] = 100.0
    u = [0.5, 0.0, 0.99, 0.7, 0.6, 0.9, 0.123, 0.99999994]
    code, token = check_sample(ctx, x, u, "f32")
    assert code == 0 and token[0] == -1
    assert check_sample(ctx, x, u, "f32", p=[0.9] * 8, k=[50] * 8)[0] == 0
    assert check_sample(ctx, x, u, "f32", T=[1e-30] * 8)[0] == 0
    assert check_sample(ctx, x, u, "f32", T=[1e30] * 8, p=[0.5] * 8)[0] == 0


@pytest.mark.parametrize("type_", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("v", [40, 3000, 50021])
def test_sample_limits_among_infinite_logits(ctx, type_, v):
    """Several logits of +infinity, of which top-p or top-k leaves the first ones: none beyond the last that stays counts."""
    rng = np.random.default_rng(v)
    n = 12
    x = rng.normal(0, 3, (n, v))
    for i in range(n):
        x[i, rng.permutation(v)[:(2, 5, v // 3, v - 1)[i % 4]]] = np.inf
    x[3, 0] = -np.inf
    u = rng.random(n)
    p = np.array([0.4, 0.3, 0.7, 0.5, 0.999, 0.01, 0.25, 0.9, 0.6, 0.8, 0.35, 0.0])
    assert check_sample(ctx, x, u, type_, p=p)[0] == 0
    assert check_sample(ctx, x, u, type_, T=rng.uniform(0.4, 2, n), k=np.minimum(v - 1, 400) + np.arange(n), p=p)[0] == 0
    assert check_sample(ctx, x, u, type_, k=[1, 3, v // 4, 2, 1, 4, 1, v // 2, 1, 2, 7, v - 2], mp=[0.0, 0.1, 1.0] * 4)[0] == 0
    assert check_sample(ctx, x, u, type_, mp=[0.5] * n, T=[0.0, 1.0] * 6)[0] == 0


def test_sample_no_numbers_and_settings_out_of_range(ctx):
    rng = np.random.default_rng(5)
    x = rng.normal(0, 2, (4, 700))
    for type_ in ("f32", "bf16", "f16"):
        y = x.copy()
        y[1, 300] = np.nan
        y[2, :] = np.nan
        assert check_sample(ctx, y, [0.2, 0.5, 0.7, 0.9], type_)[0] == -1
    import torch
    for bad in (dict(T=[-1.0, 1, 1, 1]), dict(T=[np.nan, 1, 1, 1]), dict(T=[np.inf, 1, 1, 1]), dict(p=[np.nan, 1, 1, 1]),
                dict(mp=[1.5, 0, 0, 0]), dict(mp=[-0.1, 0, 0, 0]), dict(u=[1.0, .5, .5, .5]), dict(u=[-.5, .5, .5, .5]), dict(u=[np.nan, .5, .5, .5])):
        f = lambda n, d: sh.dev(np.asarray(bad.get(n, [d] * 4), np.float32))  # noqa: E731
        token, kept, logprob = torch.full((4,), -7, dtype=torch.int32, device="cuda:0"), torch.full((4,), -7, dtype=torch.int32, device="cuda:0"), torch.zeros(4, device="cuda:0")
        ctx.hx_sample(sh.dev(x.astype(np.float32)), f("u", 0.5), token, temperature=f("T", 1.0), top_p=f("p", 1.0), min_p=f("mp", 0.0), logprob=logprob, n_kept=kept)
        assert status(ctx) == -1
        assert int(token[0]) == -1 and int(kept[0]) == 0 and float(logprob[0]) == -np.inf and int(token[1]) >= 0 and int(kept[1]) == 700


@pytest.mark.parametrize("type_", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("v", [9, 700, 5000, 40001])
def test_sample_where_few_can_stay(ctx, type_, v):
    """top-k around what is looked at in one place, ties across its end, barred and infinite logits, min-p alone."""
    rng = np.random.default_rng(v + 1)
    n = 16
    x = rng.normal(0, 3, (n, v))
    x[1] = np.round(x[1])                                      # many equal
    x[2] = 1.5
    x[3, rng.random(v) < 0.97] = -np.inf                       # fewer than k are left
    x[4, : v // 2] = -np.inf
    x[5, rng.integers(0, v, 4)] = np.inf
    x[6] = np.linspace(-9, 9, v)
    x[7] = -np.abs(x[7]) - 1000.0
    k = np.array([1, 30, 320, 50, 200, 3, 319, 64, 321, 511, 512, 2, 320, 100, 7, 40])
    p = np.where(np.arange(n) % 3 == 0, 1.0, rng.uniform(0.1, 0.99, n))
    mp = np.where(np.arange(n) % 2 == 0, 0.0, rng.uniform(0.0, 0.3, n))
    u = rng.random(n)
    T = rng.uniform(0.4, 2.0, n)
    for pad in (0, 1):
        assert check_sample(ctx, x, u, type_, T=T, k=k, p=p, mp=mp, pad=pad)[0] == 0
    assert check_sample(ctx, x, u, type_, k=k)[0] == 0
    assert check_sample(ctx, x, u, type_, T=T, mp=np.full(n, 0.02))[0] == 0
    assert check_sample(ctx, x, u, type_, T=T, mp=rng.uniform(0, 1e-12, n))[0] == 0
    y = x.copy()
    y[:, v // 3] = np.nan
    assert check_sample(ctx, y, u, type_, T=T, k=k, p=p)[0] == -1


def test_sample_of_a_negative_zero(ctx):
    rng = np.random.default_rng(9)
    x = rng.normal(0, 2, (3, 900))
    x[:, :4] = -np.inf
    for type_ in ("f32", "bf16"):
        assert check_sample(ctx, x, [-0.0] * 3, type_, p=[-0.0, 0.9, 1.0], mp=[-0.0] * 3)[0] == 0
        assert check_sample(ctx, x, [-0.0] * 3, type_, T=[-0.0, 1.0, 0.5])[0] == 0


def test_sample_many_rows_and_a_large_vocabulary(ctx):
    rng = np.random.default_rng(6)
    x = rng.normal(0, 3, (3, 262147))
    assert check_sample(ctx, x, [0.1, 0.5, 0.95], "bf16", T=[0.7, 1.0, 1.3], k=[0, 40000, 0], p=[0.97, 0.9, 1.0])[0] == 0
    x = rng.normal(0, 3, (700, 129))
    assert check_sample(ctx, x, rng.random(700), "f16", T=rng.uniform(0.2, 2, 700), p=rng.uniform(0.1, 1, 700))[0] == 0


# ---- together ------------------------------------------------------------------------------------------------------------

def test_calls_on_a_stream_of_their_own_and_captured(ctx):
    """A decode step -- room, keys and values, attention, a token -- recorded once and replayed, against the same calls made one by one."""
    import torch
    T, heads, group, dim, v = 8, 2, 2, 64, 500
    model, pool, seqs = make_cache(20, [21, 5, 64], T, layers=1, heads=heads, dim=dim, rows=3, max_pages=40, spare=60)
    g = torch.Generator().manual_seed(3)
    new = torch.randn(3, heads * (group + 2), dim, generator=g).to(torch.bfloat16).cuda()
    w = torch.randn(heads * group * dim, v, generator=g).cuda() * 0.1
    u = torch.tensor([0.1, 0.6, 0.8], device="cuda:0")
    row, one, ptr = sh.i32([2, 0, 1]), sh.i32([1, 1, 1]), sh.i32([0, 1, 2, 3])
    out, token = torch.empty(3, heads * group, dim, dtype=torch.bfloat16, device="cuda:0"), torch.empty(3, dtype=torch.int32, device="cuda:0")
    logits = torch.empty(3, v, device="cuda:0")

    def step():
        ctx.hx_kv_grow(pool, seqs, row, one)
        ctx.hx_kv_write(pool, 0, seqs, row, ptr, new[:, heads * group:heads * (group + 1)], new[:, heads * (group + 1):])
        ctx.hx_attend(pool, 0, seqs, ptr, new[:, :heads * group], out, max_q=1, row=row, window=24, n_sink=2)
        torch.mm(out.reshape(3, -1).float(), w, out=logits)
        ctx.hx_sample(logits, u, token, top_p=u)
    state = [pool["k"], pool["v"], pool["ref"], seqs["table"], seqs["len"]]
    begin = [x.clone() for x in state]
    step()
    want = []
    for x, y in zip(state, begin):
        x.copy_(y)
    for _ in range(12):
        step()
        torch.cuda.synchronize()
        want.append([x.clone() for x in state + [out, token]])
    for x, y in zip(state, begin):
        x.copy_(y)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    for x, y in zip(state, begin):
        x.copy_(y)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        step()
    for i in range(12):
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(state + [out, token], want[i]):
            assert torch.equal(a, b)
        torch.randn(1000, device="cuda:0").sum()             # the program's own work in between
    assert status(ctx) == 0


def test_the_example_runs(monkeypatch, capsys):
    import os
    import sys
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    monkeypatch.syspath_prepend(os.path.join(root, "examples"))
    import decode_instance
    inst, answers = decode_instance.main(["--steps", "4", "--prompt", "300", "--window", "64"])
    assert [len(x) for x in answers] == [5] * 4 and all(0 <= t < decode_instance.VOCAB for x in answers for t in x)
    # four rows of their own pages now, the prompt's gone from all windows: what is in use is what the tables hold, at the pool's start
    table, ref = inst.seqs["table"].cpu().numpy(), inst.pool["ref"].cpu().numpy()
    held = np.bincount(table[table >= 0], minlength=len(ref))
    assert np.array_equal(held, ref) and (ref[:int((ref > 0).sum())] > 0).all()
    assert (inst.seqs["len"][1:5].cpu().numpy() >= 304).all() and int(inst.seqs["len"][0]) == 0
    inst.ctx.close()
    del sys.modules["decode_instance"]
