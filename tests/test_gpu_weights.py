"""The weights that attention has given tokens go where the page calls take the tokens: against plain rules, and over steps of a decode loop that drafts."""
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


def cache(seed, lens, T, room=1, behind=np.nan, **more):
    """A cache with weights: spread numbers for its tokens, `behind` their rows' ends and in rows of no sequence."""
    c = lh.Cache(seed, lens, T, 2, 32, "bf16", layers=1, room=room, garbage=False, **more)
    w = np.full((c.rows, c.table.shape[1] * T), behind, np.float32)
    for i, n in enumerate(lens):
        w[c.where[i], :n] = np.random.default_rng(seed + i).random(n).astype(np.float32) + 0.5
    c.seqs["weight"] = sh.dev(w)
    return c, w


def same(c, w):
    assert np.array_equal(c.seqs["weight"].cpu().numpy(), w, equal_nan=True)


@pytest.mark.parametrize("T", [1, 16, 64])
def test_copies_have_their_sources_weights(ctx, T):
    lens = [5000, 33, 2 * T, 1, 0]
    c, w = cache(1, lens, T, extra_rows=7, spare=10)
    r, free = [int(x) for x in c.where], [x for x in range(c.rows) if x not in c.where]
    src, dst = [r[0], r[0], r[1], r[2], r[3], r[4], r[1], 99, r[1]], [free[0], free[1], free[2], free[3], free[4], free[5], r[2], free[6], free[2]]
    tok = [5000, 2049, 17, 2 * T, 1, 0, 5, 1, 3]                     # onto a row that is not empty, from none, onto one twice
    ctx.hx_kv_fork(c.pool, c.seqs, sh.i32(src), sh.i32(dst), sh.i32(tok))
    assert lh.status(ctx) == -6
    for s, d, t in list(zip(src, dst, tok))[:6]:
        w[d, :t] = w[s, :t]
    same(c, w)


def test_a_copy_for_which_no_page_is_left_has_none(ctx):
    c, w = cache(2, [40, 24], 16, extra_rows=3, spare=1)
    r, free = [int(x) for x in c.where], [x for x in range(c.rows) if x not in c.where]
    ctx.hx_kv_fork(c.pool, c.seqs, sh.i32([r[0], r[1]]), sh.i32(free[:2]))
    assert lh.status(ctx) == -4
    w[free[0], :40] = w[r[0], :40]
    same(c, w)


@pytest.mark.parametrize("T", [1, 16, 256])
def test_tokens_that_come_in_weigh_nothing(ctx, T):
    lens, new = [100, 0, 7, 33, 600, 16, 2], [5, 3000, 1, 0, 300, -1, 9000]
    c, w = cache(3, lens, T, room=3000 // T + 2, spare=3500 // T + 8)
    rows = [int(x) for x in c.where]
    ctx.hx_kv_grow(c.pool, c.seqs, sh.i32(rows + [rows[0], -1]), sh.i32(new + [2, 1]))      # a row listed again; more than a row can hold; fewer than none
    assert lh.status(ctx) == -6
    for i in range(5):
        w[rows[i], lens[i]:lens[i] + new[i]] = 0.0
        assert int(c.seqs["len"][rows[i]]) == lens[i] + new[i]
    same(c, w)


def test_rows_that_get_no_pages_keep_their_weights(ctx):
    c, w = cache(4, [32, 30, 31, 16], 16, room=4, spare=2)
    rows = [int(x) for x in c.where]
    ctx.hx_kv_grow(c.pool, c.seqs, sh.i32(rows), sh.i32([20, 10, 1, 1]))      # two pages, then none is left; the third needs none
    assert lh.status(ctx) == -4
    w[rows[0], 32:52], w[rows[2], 31] = 0.0, 0.0
    assert c.seqs["len"][c.seqs["len"].new_tensor(rows).long()].tolist() == [52, 30, 32, 16]
    same(c, w)


@pytest.mark.parametrize("T", [1, 16, 64])
def test_kept_tokens_take_their_weights_along(ctx, T):
    rng = np.random.default_rng(5)
    lens, drafts = [100, 33, 64, 9000, 12, 80], [32, 33, 17, 8500, 5, 0]
    c, w = cache(5, lens, T)
    rows = [int(x) for x in c.where]
    keep = [np.sort(rng.choice(d, m, replace=False)) for d, m in zip(drafts, (6, 1, 0, 5000, 5, 0))]
    more = [np.array([3, 2]), np.array([0])]                                  # falling numbers; a row listed again
    ptr = np.concatenate([[0], np.cumsum([len(k) for k in keep + more])])
    ctx.hx_kv_keep(c.pool, c.seqs, sh.i32(rows[:4] + rows[5:] + rows[4:5] + [rows[1]]), sh.i32(drafts[:4] + drafts[5:] + [5, 33]),
                   sh.i32(np.concatenate([[0], np.cumsum([len(k) for k in keep[:4] + keep[5:] + more])])),
                   sh.i32(np.concatenate(keep[:4] + keep[5:] + more)))
    assert lh.status(ctx) == -6 and len(ptr) == 9
    for i in (0, 2, 3, 5):
        base = lens[i] - drafts[i]
        m = base + len(keep[i])
        w[rows[i], base:m] = w[rows[i], base + keep[i]]
        w[rows[i], m:lens[i]] = 0.0
        assert int(c.seqs["len"][rows[i]]) == m
    base = lens[1] - drafts[1]
    w[rows[1], base:base + 1] = w[rows[1], base + keep[1]]
    w[rows[1], base + 1:lens[1]] = 0.0
    same(c, w)                                                                # the row with falling numbers as it was


def test_without_weights_given_they_stay(ctx):
    """Calls over the same tables without them: as they were, in their places."""
    c, w = cache(6, [40, 20], 16, extra_rows=2, room=3)
    r = [int(x) for x in c.where]
    empty = int(np.setdiff1d(np.arange(c.rows), c.where)[0])
    plain = {x: y for x, y in c.seqs.items() if x != "weight"}
    ctx.hx_kv_fork(c.pool, plain, sh.i32(r[:1]), sh.i32([empty]))
    ctx.hx_kv_grow(c.pool, plain, sh.i32(r[1:]), sh.i32([9]))
    ctx.hx_kv_keep(c.pool, plain, sh.i32(r[:1]), sh.i32([20]), sh.i32([0, 1]), sh.i32([7]))
    assert lh.status(ctx) == -6                                                # its tokens would move within a page that the copy holds too
    ctx.hx_kv_keep(c.pool, plain, sh.i32(r[1:]), sh.i32([20]), sh.i32([0, 1]), sh.i32([7]))
    ctx.hx_kv_free(c.pool, c.seqs, sh.i32(r[1:]))
    ctx.hx_kv_compact(c.pool, c.seqs)
    assert lh.status(ctx) == 0
    same(c, w)


def test_weights_of_other_sizes_and_of_another_array(ctx):
    from paper_2605_16637_amd import binding
    c, w = cache(7, [40, 20], 16)
    rows = sh.i32(c.where)
    short = dict(c.seqs, weight=c.seqs["weight"].flatten()[:-1])
    with pytest.raises(ValueError, match="elements"):
        ctx.hx_kv_grow(c.pool, short, rows, sh.i32([1, 1]))
    with pytest.raises(ValueError, match="pool"):
        binding.make_kv_seqs(c.seqs)
    with pytest.raises(binding.HxError, match="own"):
        ctx.hx_kv_evict(c.pool, c.seqs, rows, c.seqs["weight"].clone(), 5)
    ctx.hx_kv_evict(c.pool, c.seqs, rows, c.seqs["weight"], 50)
    assert lh.status(ctx) == 0
    same(c, w)


@pytest.mark.parametrize("window,sinks", [(0, 0), (40, 3)])
def test_a_decode_loop_that_drafts_weighs_and_evicts(ctx, window, sinks):
    """Trees of drafts come in, are weighed, and the accepted path stays: every token's weight is the sum of what it was given, whatever was drafted in its
    place.  Between the steps a call ends, its row begins again as a copy of another; at the end rows are cut by their weights."""
    import torch
    heads, group, dim, T, n, nd, steps = 2, 2, 64, 8, 3, 9, 12
    lens = [70, 33, 8]
    c = lh.Cache(8, lens, T, heads, dim, "bf16", layers=1, room=30, spare=60, garbage=False)
    c.seqs["weight"] = torch.full((c.rows, c.table.shape[1] * T), float("nan"), device="cuda:0")
    row_of = [int(x) for x in c.where]
    for i in range(n):
        c.seqs["weight"][row_of[i], :lens[i]] = 0.0                            # the prompts' tokens
    rng = np.random.default_rng(9)
    g = torch.Generator("cuda:0").manual_seed(0)
    keys = [c.of(c.k, 0, i) for i in range(n)]
    total, near = [np.zeros(x) for x in lens], [np.zeros(x) for x in lens]
    for step in range(steps):
        rows, ptr = sh.i32(row_of), sh.i32(np.arange(n + 1) * nd)
        parents = [[int(rng.integers(-1, i)) for i in range(nd)] for _ in range(n)]
        k, v = (torch.randn(n * nd, heads, dim, generator=g, device="cuda:0").bfloat16() for _ in range(2))
        q = 2 * torch.randn(n * nd, heads * group, dim, generator=g, device="cuda:0").bfloat16()
        out, lse = torch.zeros_like(q), torch.zeros(n * nd, heads * group, device="cuda:0")
        call = dict(max_q=nd, row=rows, parent=sh.i32(np.concatenate(parents)), window=window, n_sink=sinks)
        ctx.hx_kv_grow(c.pool, c.seqs, rows, sh.i32([nd] * n))
        ctx.hx_kv_write(c.pool, 0, c.seqs, rows, ptr, k, v)
        ctx.hx_attend(c.pool, 0, c.seqs, ptr, q, out, lse=lse, **call)
        ctx.hx_kv_weigh(c.pool, 0, c.seqs, ptr, q, lse, c.seqs["weight"], **call)
        paths = []
        for i in range(n):
            at, path = int(rng.integers(0, nd)), []
            while at >= 0:
                path.insert(0, at)
                at = parents[i][at]
            paths.append(path)
        ctx.hx_kv_keep(c.pool, c.seqs, rows, sh.i32([nd] * n), sh.i32(np.concatenate([[0], np.cumsum([len(p) for p in paths])])), sh.i32(np.concatenate(paths)))
        assert lh.status(ctx) == 0
        for i in range(n):
            mine = slice(i * nd, (i + 1) * nd)
            keys[i] = np.concatenate([keys[i], lh.f64(k)[mine]])
            m = len(keys[i])
            total[i], near[i] = (np.append(x, np.zeros(nd)) for x in (total[i], near[i]))
            see = sh.visible(m, nd, parents[i], window, sinks)
            for a in range(heads * group):
                x, kk, l = lh.f64(q)[mine, a], keys[i][:, a // group], lh.f64(lse)[mine, a][:, None]
                s = dim ** -0.5 * (x @ kk.T)
                w = np.where(see, np.exp(s - l), 0.0)
                # scores are dim products and as many sums in 32 bits; their difference from lse and the exponent's argument a rounding each
                off = (dim + 8) * 2.0 ** -24 * dim ** -0.5 * (np.abs(x) @ np.abs(kk).T) + 2.0 ** -22 * (2 + np.abs(s) + np.abs(l))
                total[i] += w.sum(0)
                near[i] += (w * off).sum(0)
            near[i] += (nd * heads * group + 8) * 2.0 ** -24 * total[i]
            stay = [*range(m - nd), *(m - nd + np.array(paths[i]))]
            keys[i], total[i], near[i] = keys[i][stay], total[i][stay], near[i][stay]
            got = lh.f64(c.seqs["weight"])[row_of[i], :len(stay)]
            assert int(c.seqs["len"][row_of[i]]) == len(stay)
            assert (np.abs(got - total[i]) <= near[i]).all(), (step, i, np.abs(got - total[i]).max())
        if step % 4 == 3:                                                      # one ends, and begins again from another's first tokens
            over, other = step // 4 % n, (step // 4 + 1) % n
            t = len(total[other]) - 5
            ctx.hx_kv_free(c.pool, c.seqs, sh.i32([row_of[over]]))
            ctx.hx_kv_fork(c.pool, c.seqs, sh.i32([row_of[other]]), sh.i32([row_of[over]]), sh.i32([t]))
            keys[over], total[over], near[over] = keys[other][:t], total[other][:t], near[other][:t]
    budget = max(len(x) for x in total) // 2
    kept = torch.zeros(n, budget, dtype=torch.int32, device="cuda:0")
    was = lh.f64(c.seqs["weight"])
    ctx.hx_kv_evict(c.pool, c.seqs, sh.i32(row_of), c.seqs["weight"], budget, n_first=2, n_last=6, kept=kept)
    assert lh.status(ctx) == 0
    cut = 0
    for i in range(n):
        m = len(total[i])
        if m <= budget:
            continue
        cut += 1
        stay = kept[i].tolist()
        assert np.array_equal(lh.f64(c.seqs["weight"])[row_of[i], :budget], was[row_of[i], stay])
        inner, others = [y for y in stay if 2 <= y < m - 6], np.setdiff1d(np.arange(2, m - 6), stay)
        assert total[i][others].max() <= total[i][inner].min() + near[i].max()
    assert cut > 0


def test_captured(ctx):
    import torch
    c, w = cache(10, [100, 40, 77], 16, extra_rows=2, room=4, spare=20)
    rows = sh.i32(c.where)
    empty = sh.i32(np.setdiff1d(np.arange(c.rows), c.where)[:1])
    state = [c.seqs["table"], c.seqs["len"], c.pool["ref"], c.pool["k"], c.pool["v"], c.seqs["weight"]]
    was = [t.clone() for t in state]
    drafts, ptr, keep, tok = sh.i32([20, 20, 20]), sh.i32([0, 3, 4, 4]), sh.i32([1, 5, 19, 7]), sh.i32([90])

    def calls(s):
        ctx.hx_kv_grow(c.pool, c.seqs, rows, drafts, stream=s)
        ctx.hx_kv_keep(c.pool, c.seqs, rows, drafts, ptr, keep, stream=s)
        ctx.hx_kv_fork(c.pool, c.seqs, rows[:1], empty, tok, stream=s)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    calls(s)
    s.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        calls(s)
    for seed in range(3):
        was[5] = torch.rand(state[5].shape, generator=torch.Generator("cuda:0").manual_seed(seed), device="cuda:0")
        got = []
        for call in (graph.replay, lambda: calls(None)):
            for t, x in zip(state, was):
                t.copy_(x)
            torch.cuda.synchronize()
            call()
            torch.cuda.synchronize()
            got.append([t.clone() for t in state])
        assert all(torch.equal(a, b) for a, b in zip(*got)) and lh.status(ctx) == 0
        want, old = got[0][5].cpu().numpy(), was[5].cpu().numpy()
        r = [int(x) for x in c.where]
        assert (want[r[0], 100:103] == 0).all() and np.array_equal(want[r[0], :100], old[r[0], :100])
        assert np.array_equal(want[int(empty[0]), :90], old[r[0], :90])
