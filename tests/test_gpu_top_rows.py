"""Attention over chosen pages where rows have fewer entries than a query sees in any case: tables between other tables, lengths that are said too short, budgets beyond
the rows."""
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


def check(ctx, c, lens, n_pages, n_first, n_last, max_len=None, around=0):
    """One query a sequence against the plain form; the table a slice of a larger one, in which `around` rows of no page's number lie on either side."""
    import torch
    heads, group, dim, T = 2, 2, 64, c.T
    ctx.hx_kv_bound(c.pool, 1, c.seqs, sh.i32(c.where))
    large = torch.full((c.rows + 2 * around, c.table.shape[1]), 2 ** 31 - 1, dtype=torch.int32, device="cuda:0")
    table = large[around:around + c.rows]
    table.copy_(c.seqs["table"])
    q = lh.queries(len(lens), heads * group, dim, "bf16", n_pages)
    out, lse = torch.full_like(q, 7.0), torch.full((len(lens), heads * group), 7.0, device="cuda:0")
    chosen = torch.full((len(lens), heads, n_pages), 7, dtype=torch.int32, device="cuda:0")
    ctx.hx_attend_top(c.pool, 1, dict(table=table, len=c.seqs["len"]), sh.i32(range(len(lens) + 1)), q, out, max_q=1, max_len=max_len, n_pages=n_pages,
                      n_first=n_first, n_last=n_last, row=sh.i32(c.where), chosen=chosen, lse=lse)
    assert lh.status(ctx) == 0
    qf, got, got_lse, bounds = lh.f64(q), lh.f64(out), lh.f64(lse), lh.f64(c.pool["bounds"])
    for i, n in enumerate(lens):
        k, v, pages = c.of(c.k, 1, i), c.of(c.v, 1, i), c.table[c.where[i], :c.need[i]]
        for h in range(heads):
            part = slice(h * group, (h + 1) * group)
            want = lh.choose(bounds[1, np.maximum(pages, 0), h], pages >= 0, (n - 1) // T, qf[i, part], 1.0, n_pages, n_first, n_last)
            assert chosen[i, h].tolist() == want + [-1] * (n_pages - len(want)), (i, h)
            see = np.isin(np.arange(n) // T, want)
            lh.compare(got[i:i + 1, part], got_lse[i:i + 1, part], qf[i:i + 1, part], k[:, h:h + 1], v[:, h:h + 1], see[None], dim ** -0.5, group, "bf16")


@pytest.mark.parametrize("n_pages,n_first,n_last", [(8, 4, 4), (9, 0, 5), (9, 8, 1), (40, 4, 36), (4096, 4000, 96), (4, 0, 4), (5, 4, 1)])
@pytest.mark.parametrize("max_len", [None, 1])
def test_rows_shorter_than_what_is_seen_in_any_case(ctx, n_pages, n_first, n_last, max_len):
    """Rows of one to three pages, the tables' first and last among them, where no row has more entries than are seen."""
    lens = [1, 8, 9, 16, 17, 24]
    c = lh.Cache(n_pages, lens, 8, 2, 64, "bf16", bounds=True, extra_rows=0, room=0, missing=[(3, 0)])
    check(ctx, c, lens, n_pages, n_first, n_last, max_len, around=5000)


@pytest.mark.parametrize("n_pages,n_first,n_last", [(12, 5, 7), (7, 1, 5), (9, 8, 1)])
@pytest.mark.parametrize("max_len", [1, 100])
def test_short_rows_beside_long_ones_of_which_less_is_said(ctx, n_pages, n_first, n_last, max_len):
    """Rows that are longer than max_len have their entries looked up again; short ones beside them have none there."""
    lens = [1, 2300, 9, 130, 96, 97]
    c = lh.Cache(n_pages, lens, 8, 2, 64, "bf16", bounds=True, extra_rows=0, room=0, missing=[(1, 0), (1, 200)])
    check(ctx, c, lens, n_pages, n_first, n_last, max_len, around=40)


def test_pages_beyond_a_row_take_no_room():
    """65536 queries and heads over rows of two entries: a budget of 4096 pages is one of two."""
    import torch
    from paper_2605_16637_amd import binding
    fresh = binding.Context(0)
    n = 8192
    c = lh.Cache(51, [16, 9], 8, 8, 64, "bf16", bounds=True, extra_rows=0, room=0)
    fresh.hx_kv_bound(c.pool, 1, c.seqs, sh.i32(c.where))
    q = lh.queries(n, 8, 64, "bf16", 0)
    out, want = torch.zeros(2, n, 8, 64, dtype=torch.bfloat16, device="cuda:0")
    chosen = torch.full((n, 8, 4096), 7, dtype=torch.int32, device="cuda:0")
    few = torch.full((n, 8, 2), 7, dtype=torch.int32, device="cuda:0")
    call = dict(max_q=1, row=sh.i32(np.resize(c.where, n)))
    ptr = sh.i32(range(n + 1))
    torch.cuda.synchronize()
    before = torch.cuda.mem_get_info()[0]
    fresh.hx_attend_top(c.pool, 1, c.seqs, ptr, q, out, n_pages=4096, n_first=4000, n_last=90, chosen=chosen, **call)
    torch.cuda.synchronize()
    assert before - torch.cuda.mem_get_info()[0] < 128 << 20
    fresh.hx_attend_top(c.pool, 1, c.seqs, ptr, q, want, n_pages=2, n_last=2, chosen=few, **call)
    assert lh.status(fresh) == 0 and torch.equal(out, want)
    assert torch.equal(chosen[:, :, :2], few) and bool((chosen[:, :, 2:] == -1).all()) and bool((few == sh.i32([0, 1])).all())
    fresh.close()


def test_queries_that_see_all_pages_in_several_parts():
    """So many chosen pages that not all queries' are held at once, where there are no scores."""
    import torch
    from paper_2605_16637_amd import binding
    fresh = binding.Context(0)
    n, heads, n_q = 4096, 16, 1100                              # 1023 queries' pages are 256 MB
    c = lh.Cache(52, [n], 1, heads, 64, "bf16", bounds=True, extra_rows=0, room=0, layers=1, spare=0)
    q = lh.queries(n_q, heads, 64, "bf16", 0)
    out, lse = torch.zeros_like(q), torch.zeros(n_q, heads, device="cuda:0")
    chosen = torch.full((n_q, heads, n), 7, dtype=torch.int32, device="cuda:0")
    torch.cuda.synchronize()
    before = torch.cuda.mem_get_info()[0]
    fresh.hx_attend_top(c.pool, 0, c.seqs, sh.i32([0, n_q]), q, out, max_q=n_q, n_pages=n, chosen=chosen, lse=lse)
    torch.cuda.synchronize()
    assert before - torch.cuda.mem_get_info()[0] < 1 << 30
    assert lh.status(fresh) == 0
    b = torch.arange(n, device="cuda:0", dtype=torch.int32)
    for j in range(n_q):
        assert bool((chosen[j] == torch.where(b <= n - n_q + j, b, -1)).all())
    some = [0, 1, 1021, 1022, 1023, 1024, n_q - 1]
    k, v = c.of(c.k, 0, 0), c.of(c.v, 0, 0)
    see = np.arange(n) <= n - n_q + np.asarray(some)[:, None]
    lh.compare(lh.f64(out)[some], lh.f64(lse)[some], lh.f64(q)[some], k, v, see, 64 ** -0.5, 1, "bf16")
    fresh.close()
