"""Weights that attention gives cached tokens, and the eviction of the others, against plain forms in whole numbers and 64 bits."""
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


# ---- weights ----------------------------------------------------------------------------------------------------------

def check_weigh(ctx, lens, nq, heads=2, group=2, dim=64, T=16, type_="bf16", cache=None, window=0, sinks=0, parents=None, scale=None, missing=(), wide=True,
                seed=0, max_len=None):
    import torch
    c = lh.Cache(seed, lens, T, heads, dim, cache or type_, missing=missing)
    ptr = np.concatenate([[0], np.cumsum(nq)])
    total = int(ptr[-1])
    q = lh.queries(total, heads * group, dim, type_, seed, wide)
    out, lse = torch.zeros_like(q), torch.zeros(total, heads * group, device="cuda:0")
    weight = torch.rand(c.rows, c.table.shape[1] * T, generator=torch.Generator("cuda:0").manual_seed(seed), device="cuda:0")
    was = lh.f64(weight)
    par = None if parents is None else sh.i32(np.concatenate([np.asarray(p, np.int64) for p in parents]))
    call = dict(max_q=max(nq), max_len=max_len, row=sh.i32(c.where), scale=scale, window=window, n_sink=sinks, parent=par)
    ctx.hx_attend(c.pool, 1, c.seqs, sh.i32(ptr), q, out, lse=lse, **call)
    ctx.hx_kv_weigh(c.pool, 1, c.seqs, sh.i32(ptr), q, lse, weight, **call)
    assert lh.status(ctx) == 0
    got, qf, l = lh.f64(weight), lh.f64(q), lh.f64(lse)
    scale = dim ** -0.5 if scale is None else scale
    want, near = was.copy(), 2.0 ** -24 * was
    for i in range(len(lens)):
        see = sh.visible(lens[i], nq[i], None if parents is None else parents[i], window, sinks) & c.there(i)
        k = c.of(c.k, 1, i)
        for a in range(heads * group):
            x = qf[ptr[i]:ptr[i + 1], a]
            mine = l[ptr[i]:ptr[i + 1], a][:, None]
            with np.errstate(invalid="ignore", over="ignore"):
                w = np.where(see, np.exp(scale * (x @ k[:, a // group].T) - mine), 0.0)
                # scores are dim products and as many sums in 32 bits; their difference from lse and the exponent's argument a rounding each
                off = (dim + 8) * 2.0 ** -24 * abs(scale) * (np.abs(x) @ np.abs(k[:, a // group]).T) + 2.0 ** -22 * (2 + np.abs(scale * (x @ k[:, a // group].T)) + np.abs(mine))
                r = c.where[i]
                want[r, :lens[i]] += w.sum(0)
                near[r, :lens[i]] += np.where(see, w * off, 0.0).sum(0)
    near += (sum(nq) * heads * group + 8) * 2.0 ** -24 * want
    assert (np.abs(got - want) <= near).all(), np.abs(got - want).max()
    untouched = np.ones_like(got, bool)
    for i in range(len(lens)):
        untouched[c.where[i], :lens[i]] = False
    assert np.array_equal(got[untouched], was[untouched])                     # behind the rows' ends, and other rows


@pytest.mark.parametrize("type_,cache", [("bf16", "bf16"), ("f16", "f16"), ("bf16", "e4m3"), ("f16", "e4m3"), ("bf16", "e2m1"), ("f16", "e2m1")])
@pytest.mark.parametrize("dim", [64, 128, 256])
def test_weights_of_one_query_each(ctx, type_, cache, dim):
    lens = [1, 2, 15, 16, 17, 63, 64, 65, 127, 129, 257, 700]
    check_weigh(ctx, lens, [1] * len(lens), dim=dim, type_=type_, cache=cache)


@pytest.mark.parametrize("T", [1, 2, 8, 32, 256, 1024])
def test_weights_over_page_sizes(ctx, T):
    check_weigh(ctx, [3, 100, 333, 1500], [1, 5, 40, 2], T=T, window=70, sinks=3)
    check_weigh(ctx, [3, 100, 333, 1500], [1, 5, 40, 2], T=T, seed=1, max_len=1)


@pytest.mark.parametrize("heads,group", [(1, 1), (1, 7), (3, 1), (2, 3), (1, 16), (1, 17), (2, 33), (8, 4)])
def test_weights_of_head_layouts(ctx, heads, group):
    check_weigh(ctx, [5, 90, 200], [1, 3, 2], heads=heads, group=group)


@pytest.mark.parametrize("heads,group", [(1, 1), (5, 3), (2, 7), (3, 16), (1, 17), (2, 40)])
@pytest.mark.parametrize("dim,cache", [(64, "e4m3"), (128, "bf16"), (256, "e2m1")])
@pytest.mark.parametrize("wide", [True, False])
def test_weights_of_many_rows_and_head_layouts(ctx, heads, group, dim, cache, wide):
    """Rows that end inside a block of 16, heads that end inside one, fewer blocks than wavefronts, and queries that lie anyhow."""
    check_weigh(ctx, [17, 100, 75], [17, 33, 20], heads=heads, group=group, dim=dim, cache=cache, wide=wide, seed=group)


@pytest.mark.parametrize("window,sinks", [(1, 0), (2, 1), (17, 5), (64, 70), (65, 0), (500, 1000)])
def test_weights_of_windows_and_sinks(ctx, window, sinks):
    check_weigh(ctx, [1, 40, 64, 129, 300, 411], [1] * 6, window=window, sinks=sinks)
    check_weigh(ctx, [1, 40, 64, 129, 300, 411], [1, 40, 9, 70, 150, 33], group=3, heads=1, window=window, sinks=sinks, seed=1)


@pytest.mark.parametrize("n", [1, 8, 25, 256])
@pytest.mark.parametrize("window,sinks", [(0, 0), (20, 2)])
def test_weights_of_trees(ctx, n, window, sinks):
    rng = np.random.default_rng(n)
    parents = [[int(rng.integers(max(-1, i - near), i)) for i in range(n)] for near in (1, 4, 300)]
    for p in parents:
        if n > 10:
            p[-2:] = [-2, -2]
    check_weigh(ctx, [n, n + 1, n + 333], [n] * 3, heads=1, group=3, dim=128, window=window, sinks=sinks, parents=parents)


@pytest.mark.parametrize("dim,cache", [(64, "f16"), (256, "f16"), (256, "e4m3")])
def test_weights_of_trees_over_head_sizes(ctx, dim, cache):
    """The trees' words beside the most rows in LDS that there are."""
    rng = np.random.default_rng(dim)
    n = 40
    parents = [[int(rng.integers(max(-1, i - 9), i)) for i in range(n)] for _ in range(2)]
    check_weigh(ctx, [n, n + 210], [n] * 2, heads=2, group=5, dim=dim, type_="f16", cache=cache, parents=parents, wide=dim == 64)


def test_weights_where_pages_are_not_there_strides_and_scales(ctx):
    check_weigh(ctx, [40, 64, 300, 16], [1, 1, 60, 1], missing=[(0, 0), (1, 1), (2, 5), (3, 0)])
    check_weigh(ctx, [40, 64, 300, 16], [3, 60, 20, 1], wide=False, T=8)
    for scale in (0.0, -0.3, 2.0):
        check_weigh(ctx, [100, 50], [1, 40], scale=scale)


def test_a_query_without_a_finite_sum_adds_nothing(ctx):
    """lse of NaN or infinity, as a query that sees a NaN or infinite key has, or none."""
    import torch
    c = lh.Cache(1, [50, 60], 16, 2, 64, "bf16")
    q = lh.queries(3, 4, 64, "bf16", 0)
    out, lse = torch.zeros_like(q), torch.zeros(3, 4, device="cuda:0")
    weight = torch.zeros(c.rows, c.table.shape[1] * 16, device="cuda:0")
    call = dict(max_q=2, row=sh.i32(c.where))
    c.pool["k"][1, c.table[c.where[0], 3], 0, 49 % 16] = float("nan")           # the last token of the first, in one head: its first query does not see it
    ctx.hx_attend(c.pool, 1, c.seqs, sh.i32([0, 2, 3]), q, out, lse=lse, **call)
    assert bool(lse[1, :2].isnan().all()) and bool(lse[[0, 2]].isfinite().all())
    lse[2, 3] = float("inf")
    ctx.hx_kv_weigh(c.pool, 1, c.seqs, sh.i32([0, 2, 3]), q, lse, weight, **call)
    assert lh.status(ctx) == 0 and bool(weight.isfinite().all())
    # each query and head with a sum has given 1 in all
    assert abs(float(weight[int(c.where[0])].sum()) - 6) < 1e-4 and abs(float(weight[int(c.where[1])].sum()) - 3) < 1e-4


def test_weights_of_rows_in_error(ctx):
    import torch
    c = lh.Cache(2, [50, 60, 9], 16, 2, 64, "bf16")
    r = [int(x) for x in c.where]
    q = lh.queries(6, 4, 64, "bf16", 0)
    lse = torch.full((6, 4), 5.0, device="cuda:0")
    weight, want = torch.zeros(2, c.rows, c.table.shape[1] * 16, device="cuda:0")
    rows, ptr = [r[0], 99, r[0], r[1], -1], [0, 1, 2, 3, 5, 6]                  # the third lists a row again
    ctx.hx_kv_weigh(c.pool, 1, c.seqs, sh.i32(ptr), q, lse, weight, max_q=2, row=sh.i32(rows))
    assert lh.status(ctx) == -6
    ctx.hx_kv_weigh(c.pool, 1, c.seqs, sh.i32([0, 1]), q[:1], lse[:1], want, max_q=1, row=sh.i32(r[:1]))
    ctx.hx_kv_weigh(c.pool, 1, c.seqs, sh.i32([0, 2]), q[3:5], lse[3:5], want, max_q=2, row=sh.i32(r[1:2]))
    assert lh.status(ctx) == 0 and torch.equal(weight, want) and bool((want > 0).any())
    seqs = dict(table=c.seqs["table"].clone(), len=c.seqs["len"])
    seqs["table"][r[0], 1] = c.n_pages
    weight.zero_()
    ctx.hx_kv_weigh(c.pool, 1, seqs, sh.i32([0, 1]), q[:1], lse[:1], weight, max_q=1, row=sh.i32(r[:1]))
    assert lh.status(ctx) == -6 and bool((weight[r[0], 16:32] == 0).all()) and bool((weight[r[0], :16] > 0).all())
    ctx.hx_kv_weigh(c.pool, 1, c.seqs, sh.i32([0]), q[:0], lse[:0], weight, max_q=0)
    assert lh.status(ctx) == 0


def test_weights_do_not_depend_on_timing(ctx):
    import torch
    c = lh.Cache(3, [3000, 17, 900], 16, 4, 64, "f16")
    q = lh.queries(60, 16, 64, "f16", 0)
    out, lse = torch.zeros_like(q), torch.zeros(60, 16, device="cuda:0")
    call = dict(max_q=40, row=sh.i32(c.where))
    ctx.hx_attend(c.pool, 1, c.seqs, sh.i32([0, 40, 50, 60]), q, out, lse=lse, **call)
    got = []
    for _ in range(3):
        weight = torch.zeros(c.rows, c.table.shape[1] * 16, device="cuda:0")
        ctx.hx_kv_weigh(c.pool, 1, c.seqs, sh.i32([0, 40, 50, 60]), q, lse, weight, **call)
        got.append(weight)
    assert torch.equal(got[0], got[1]) and torch.equal(got[0], got[2])


# ---- eviction ---------------------------------------------------------------------------------------------------------

class Model:
    """A cache's tables and what its pages hold, as arrays that the plain rules change."""

    def __init__(self, c):
        self.T, self.table, self.length, self.ref = c.T, c.table.copy(), c.length.copy(), c.ref.copy()
        self.pages = {x: c.pool[x].cpu().view(dtype=raw(c.pool[x])).numpy().copy() for x in ("k", "v", "k_exp", "v_exp") if x in c.pool}


def raw(t):
    import torch
    return {1: torch.uint8, 2: torch.int16}[t.element_size()]


def same(model, c):
    assert np.array_equal(c.seqs["len"].cpu().numpy(), model.length) and np.array_equal(c.seqs["table"].cpu().numpy(), model.table)
    assert np.array_equal(c.pool["ref"].cpu().numpy(), model.ref)
    for x, y in model.pages.items():
        assert np.array_equal(c.pool[x].cpu().view(dtype=raw(c.pool[x])).numpy(), y), x


def weights(c, seed, kind="spread"):
    rng = np.random.default_rng(seed)
    shape = (c.rows, c.table.shape[1] * c.T)
    w = np.exp(1.5 * rng.standard_normal(shape)) if kind == "spread" else rng.integers(0, 3, shape) if kind == "few" else np.full(shape, 0.25)
    return w.astype(np.float32)


def check_evict(ctx, c, w, rows, n_keep, n_first=0, n_last=0, code=(), with_kept=True):
    import torch
    model, weight = Model(c), sh.dev(w)
    errors, kept = lh.evict(model, w, rows, n_keep, n_first, n_last)
    got = torch.full((len(rows), n_keep), 7, dtype=torch.int32, device="cuda:0") if with_kept else None
    ctx.hx_kv_evict(c.pool, c.seqs, sh.i32(rows), weight, n_keep=n_keep, n_first=n_first, n_last=n_last, kept=got)
    assert errors == set(code) and (lh.status(ctx) in errors if errors else lh.status(ctx) == 0)
    same(model, c)
    assert np.array_equal(weight.cpu().numpy(), w, equal_nan=True)
    if with_kept:
        for i, k in enumerate(kept):
            assert got[i].tolist() == (k or []) + [-1] * (n_keep - len(k or []))
    return model


@pytest.mark.parametrize("cache", ["bf16", "f16", "e4m3", "e2m1"])
@pytest.mark.parametrize("T", [1, 4, 16, 64])
@pytest.mark.parametrize("kind", ["spread", "few", "same"])
def test_evict_keeps_the_largest_weights(ctx, cache, T, kind):
    lens = [100, 33, 32, 1, 0, 700, 34, 65]
    c = lh.Cache(T, lens, T, 3, 64, cache, layers=2)
    rows = [int(c.where[i]) for i in (5, 0, 1, 2, 3, 4, 6, 7)]
    check_evict(ctx, c, weights(c, 1, kind), rows, 32, 2, 5)


@pytest.mark.parametrize("dim,heads", [(16, 1), (48, 5), (128, 8), (1024, 1)])
@pytest.mark.parametrize("n_keep,n_first,n_last", [(1, 0, 0), (1, 1, 0), (1, 0, 1), (64, 64, 0), (64, 0, 64), (64, 30, 34), (511, 0, 7), (257, 4, 20)])
def test_evict_budgets(ctx, dim, heads, n_keep, n_first, n_last):
    c = lh.Cache(5, [600, 512, 70], 16, heads, dim, "bf16", layers=1)
    check_evict(ctx, c, weights(c, 2), [int(x) for x in c.where], n_keep, n_first, n_last, with_kept=n_keep != 257)


def test_evict_of_long_rows(ctx):
    """More tokens than a workgroup's bins and lists hold at once, budgets of several rounds of moves, weights equal in thousands."""
    for kind, n_keep in (("spread", 3500), ("few", 5000), ("same", 2600)):
        c = lh.Cache(6, [20000, 9001], 32, 1, 32, "bf16", layers=1)
        check_evict(ctx, c, weights(c, 3, kind), [int(x) for x in c.where], n_keep, 4, 100)


def test_evict_of_shared_pages(ctx):
    """Pages that others hold too are replaced where something in them changes, the lowest free ones, in the order of the rows; the others' rows stay as they are."""
    c = lh.Cache(7, [200, 150, 90], 16, 2, 64, "bf16", spare=30, extra_rows=4)
    r = [int(x) for x in c.where]
    free = [x for x in range(c.rows) if x not in r]
    ctx.hx_kv_fork(c.pool, c.seqs, sh.i32([r[0], r[1], r[0]]), sh.i32(free[:3]), sh.i32([200, 150, 64]))
    c.table, c.length, c.ref = (x.cpu().numpy().astype(np.int64) for x in (c.seqs["table"], c.seqs["len"], c.pool["ref"]))
    w = weights(c, 4)
    model = check_evict(ctx, c, w, [r[1], r[0], free[1]], 40, 3, 10)
    assert model.ref.min() >= 0
    # a row that keeps its first tokens alone: a page that it shares and goes on in is replaced though nothing in it moves
    c.table, c.length, c.ref = (x.cpu().numpy().astype(np.int64) for x in (c.seqs["table"], c.seqs["len"], c.pool["ref"]))
    w = np.zeros_like(w)
    w[free[0], :24] = 1.0
    check_evict(ctx, c, w, [free[0]], 24)
    c.table, c.length, c.ref = (x.cpu().numpy().astype(np.int64) for x in (c.seqs["table"], c.seqs["len"], c.pool["ref"]))
    w[free[2], :32] = 1.0
    check_evict(ctx, c, w, [free[2]], 32)                       # and full ones stay shared


def test_evict_without_a_page_left(ctx):
    c = lh.Cache(8, [100, 100, 100], 16, 2, 64, "bf16", spare=3, extra_rows=3)
    r = [int(x) for x in c.where]
    free = [x for x in range(c.rows) if x not in r]
    ctx.hx_kv_fork(c.pool, c.seqs, sh.i32(r[:2]), sh.i32(free[:2]), sh.i32([96, 96]))
    c.table, c.length, c.ref = (x.cpu().numpy().astype(np.int64) for x in (c.seqs["table"], c.seqs["len"], c.pool["ref"]))
    check_evict(ctx, c, weights(c, 5), [r[0], r[1], r[2]], 40, code=[-4])        # three pages each where three are left: the second stays as it is


def test_evict_of_rows_with_holes(ctx):
    """Tokens whose pages are gone go; entries without a page get one where tokens move there; a row may become empty."""
    missing = [(0, 0), (0, 3), (1, 1), (1, 2), (1, 3), (2, 0), (2, 1), (2, 2), (3, 4)]
    c = lh.Cache(9, [100, 80, 40, 70, 64], 16, 2, 64, "bf16", missing=missing)
    w = weights(c, 6)
    w[int(c.where[4]), 3] = np.nan
    w[int(c.where[4]), 9] = -1.0
    w[int(c.where[4]), 11] = np.inf
    check_evict(ctx, c, w, [int(x) for x in c.where], 30, 5, 8)


def test_evict_of_rows_in_error(ctx):
    c = lh.Cache(10, [100, 50, 60], 16, 2, 64, "bf16")
    r = [int(x) for x in c.where]
    c.length[r[2]] = c.table.shape[1] * 16 + 1
    c.seqs["len"][r[2]] = c.table.shape[1] * 16 + 1
    check_evict(ctx, c, weights(c, 7), [r[0], 99, -1, r[0], r[2], r[1]], 20, 1, 1, code=[-6])
    ctx.hx_kv_evict(c.pool, c.seqs, sh.i32([]), sh.dev(weights(c, 7)), n_keep=5)
    assert lh.status(ctx) == 0


def test_a_decode_loop_that_keeps_its_budget(ctx):
    """Tokens come in, are attended to, weighed, and the row is cut when it is over its budget; bounds taken again.  Every step's output equals
    attention over what has stayed."""
    import torch
    heads, group, dim, T, budget, steps, n0 = 2, 2, 64, 8, 48, 40, 70
    c = lh.Cache(11, [n0, n0 - 9], T, heads, dim, "e2m1", layers=1, spare=40, room=20, bounds=True, garbage=False)
    rows, n = sh.i32(c.where), 2
    weight = torch.zeros(c.rows, c.table.shape[1] * T, device="cuda:0")
    g = torch.Generator("cuda:0").manual_seed(0)
    mine = [[c.of(c.k, 0, i), c.of(c.v, 0, i)] for i in range(n)]
    total = [np.zeros(len(m[0])) for m in mine]
    kept = torch.zeros(n, budget, dtype=torch.int32, device="cuda:0")
    for step in range(steps):
        k, v = (torch.randn(n, heads, dim, generator=g, device="cuda:0").bfloat16() for _ in range(2))
        q = torch.randn(n, heads * group, dim, generator=g, device="cuda:0").bfloat16()
        out, lse, ptr = torch.zeros_like(q), torch.zeros(n, heads * group, device="cuda:0"), sh.i32(range(n + 1))
        ctx.hx_kv_grow(c.pool, c.seqs, rows, sh.i32([1] * n))
        ctx.hx_kv_write(c.pool, 0, c.seqs, rows, ptr, k, v)
        ctx.hx_attend(c.pool, 0, c.seqs, ptr, q, out, max_q=1, row=rows, lse=lse)
        ctx.hx_kv_weigh(c.pool, 0, c.seqs, ptr, q, lse, weight, max_q=1, row=rows)
        ctx.hx_kv_evict(c.pool, c.seqs, rows, weight, n_keep=budget, n_first=2, n_last=8, kept=kept)
        ctx.hx_kv_bound(c.pool, 0, c.seqs, rows)
        assert lh.status(ctx) == 0
        for i in range(n):
            for x, new in enumerate((k, v)):
                mine[i][x] = np.concatenate([mine[i][x], lh.decode(*lh.encode(lh.f64(new)[i:i + 1]))])
            total[i] = np.append(total[i], 0.0)
            lh.compare(lh.f64(out)[i:i + 1], lh.f64(lse)[i:i + 1], lh.f64(q)[i:i + 1], mine[i][0], mine[i][1], np.ones((1, len(mine[i][0])), bool), dim ** -0.5, group, "bf16")
            for a in range(heads * group):
                s = dim ** -0.5 * (mine[i][0][:, a // group] @ lh.f64(q)[i, a])
                total[i] += np.exp(s - s.max()) / np.exp(s - s.max()).sum()
            if len(total[i]) > budget:
                stay = kept[i].tolist()
                others = np.setdiff1d(np.arange(2, len(total[i]) - 8), stay)
                inner = [y for y in stay if 2 <= y < len(total[i]) - 8]
                # (weights beside the border may be told apart the other way by their own rounding)
                assert len(stay) == budget and total[i][others].max() <= total[i][inner].min() * (1 + 1e-4)
                mine[i] = [x[stay] for x in mine[i]]
                total[i] = total[i][stay]
            else:
                assert kept[i].tolist() == [-1] * budget
    assert c.seqs["len"][rows.long()].tolist() == [budget] * n
    got = lh.f64(c.pool["bounds"])
    table = c.seqs["table"].cpu().numpy()
    for i in range(n):
        for b in range(budget // T):
            want = lh.bounds_of(mine[i][0][b * T:(b + 1) * T].transpose(1, 0, 2), T)
            assert np.array_equal(got[0, table[c.where[i], b]], want)


def test_captured_and_on_another_stream(ctx):
    import torch
    c = lh.Cache(12, [300, 130], 8, 2, 64, "bf16", garbage=False)
    q, lse = lh.queries(2, 4, 64, "bf16", 0), torch.full((2, 4), 6.0, device="cuda:0")
    row, ptr = sh.i32(c.where), sh.i32([0, 1, 2])
    weight = torch.zeros(c.rows, c.table.shape[1] * 8, device="cuda:0")
    state = [c.seqs["table"], c.seqs["len"], c.pool["ref"], c.pool["k"], c.pool["v"], weight]
    was = [t.clone() for t in state]

    def calls(s):
        ctx.hx_kv_weigh(c.pool, 1, c.seqs, ptr, q, lse, weight, max_q=1, row=row, stream=s)
        ctx.hx_kv_evict(c.pool, c.seqs, row, weight, n_keep=90, n_first=4, n_last=9, stream=s)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    calls(s)
    s.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        calls(s)
    for seed in range(3):
        was[5] = torch.rand(weight.shape, generator=torch.Generator("cuda:0").manual_seed(seed), device="cuda:0")
        got = []
        for call in (graph.replay, lambda: calls(None)):
            for t, x in zip(state, was):
                t.copy_(x)
            torch.cuda.synchronize()
            call()
            torch.cuda.synchronize()
            got.append([t.clone() for t in state])
        assert all(torch.equal(a, b) for a, b in zip(*got)) and lh.status(ctx) == 0
        assert c.seqs["len"][row.long()].tolist() == [90, 90]


@pytest.mark.parametrize("cache,T,pages", [("bf16", 1, 1100000), ("e2m1", 32, 300000)])
def test_pages_past_32_bits(ctx, cache, T, pages):
    """All operators over rows whose pages lie at a pool's end, where bytes, of keys or bounds, pass 2^32: as over a small pool."""
    import torch
    heads, group, dim, lens, nq = 8, 2, 128, [40 * T // min(T, 4), 75], [1, 20]
    c = lh.Cache(31, lens, T, heads, dim, cache, layers=1, extra_rows=0, bounds=True, garbage=False)
    small, far = dict(c.pool), pages - c.n_pages
    big = {}
    for name, x in small.items():
        if name == "page_tokens":
            big[name] = x
        elif name == "ref":
            big[name] = torch.cat([torch.ones(far, dtype=torch.int32, device="cuda:0"), x])
        else:
            big[name] = torch.empty((1, pages) + tuple(x.shape[2:]), dtype=x.dtype, device="cuda:0")
            big[name][:, far:] = x
    assert max(x.numel() * x.element_size() for x in big.values() if torch.is_tensor(x)) > 2 ** 32
    got = []
    for pool, add in ((small, 0), (big, far)):
        table = c.seqs["table"].clone()
        table[table >= 0] += add
        seqs = dict(table=table, len=c.seqs["len"].clone())
        row, ptr = sh.i32(c.where), sh.i32([0, 1, 21])
        x = torch.randn(2, 21, heads, dim, device="cuda:0", generator=torch.Generator("cuda:0").manual_seed(2))
        ctx.hx_kv_write(pool, 0, seqs, row, ptr, x[0], x[1])
        ctx.hx_kv_bound(pool, 0, seqs, row)
        q = lh.queries(21, heads * group, dim, "bf16", 3)
        out, lse = torch.zeros(2, 21, heads * group, dim, dtype=torch.bfloat16, device="cuda:0"), torch.zeros(2, 21, heads * group, device="cuda:0")
        ctx.hx_attend(pool, 0, seqs, ptr, q, out[0], max_q=20, row=row, lse=lse[0])
        ctx.hx_attend_top(pool, 0, seqs, ptr, q, out[1], max_q=20, n_pages=2, row=row, lse=lse[1])
        weight = torch.zeros(c.rows, table.shape[1] * T, device="cuda:0")
        ctx.hx_kv_weigh(pool, 0, seqs, ptr, q, lse[0], weight, max_q=20, row=row)
        ctx.hx_kv_weigh(pool, 0, seqs, sh.i32([0, 1]), q, lse[0], weight, max_q=1, row=row[:1])
        kept = torch.zeros(2, 33, dtype=torch.int32, device="cuda:0")
        ctx.hx_kv_evict(pool, seqs, row, weight, 33, n_last=2, kept=kept)
        assert lh.status(ctx) == 0
        k, v = torch.zeros(2, 66, heads, dim, device="cuda:0")
        ctx.hx_kv_read(pool, 0, seqs, row, sh.i32([0, 33, 66]), k, v)
        assert lh.status(ctx) == 0 and seqs["len"][row.long()].tolist() == [33, 33]
        got.append((out, lse, weight, kept, k, v))
    for one, other in zip(*got):
        assert torch.equal(one, other)
