"""Budgets beyond what rows hold, up to the largest number, and the scratch that they take."""
import numpy as np
import pytest

from tests import long_helpers as lh
from tests import serve_helpers as sh
from tests.test_gpu_evict import Model, check_evict, same, weights

pytestmark = pytest.mark.gpu

MOST = 2 ** 31 - 1


@pytest.fixture(scope="module")
def ctx():
    from paper_2605_16637_amd import binding
    c = binding.Context(0)
    yield c
    c.close()


def cache():
    return lh.Cache(41, [100, 33, 64], 16, 2, 64, "bf16")


@pytest.mark.parametrize("n_keep,n_first,n_last", [(MOST, 0, 0), (MOST, MOST, 0), (MOST, 1, MOST - 1), (MOST - 511, 7, 9), (MOST - 512, 0, 0), (2 ** 30, 2 ** 30, 0)])
def test_budgets_beyond_every_row(ctx, n_keep, n_first, n_last):
    """Nothing is to be done, and nothing is; rows in error are told all the same."""
    c = cache()
    model, w = Model(c), weights(c, 1)
    weight = sh.dev(w)
    rows = [int(x) for x in c.where]
    ctx.hx_kv_evict(c.pool, c.seqs, sh.i32(rows), weight, n_keep, n_first, n_last)
    assert lh.status(ctx) == 0
    ctx.hx_kv_evict(c.pool, c.seqs, sh.i32([rows[0], -1, rows[0]]), weight, n_keep, n_first, n_last)
    assert lh.status(ctx) == -6
    same(model, c)
    assert np.array_equal(weight.cpu().numpy(), w)


@pytest.mark.parametrize("n_keep", [MOST, MOST - 300])
def test_positions_kept_of_the_largest_budgets(ctx, n_keep):
    """All are none, up to the last of them, and nothing beside them is written."""
    import torch
    c = cache()
    held = torch.full((n_keep + 2048,), 7, dtype=torch.int32, device="cuda:0")
    kept = held[1024:1024 + n_keep]
    ctx.hx_kv_evict(c.pool, c.seqs, sh.i32(c.where[:1]), sh.dev(weights(c, 1)), n_keep, kept=kept)
    assert lh.status(ctx) == 0
    assert bool((held[:1024] == 7).all()) and bool((held[1024 + n_keep:] == 7).all())
    assert int(kept[0]) == -1 and int(kept[-1]) == -1 and all(bool((x == -1).all()) for x in kept.split(1 << 28))


@pytest.mark.parametrize("over", [0, 1, 2])
def test_budgets_around_what_rows_can_hold(ctx, over):
    """Tables of seven pages: one token fewer than a full row, as many, one more; positions kept in the caller's own pitch."""
    lens = [112, 111, 1, 0]
    c = lh.Cache(42, lens, 16, 2, 64, "bf16", room=0, extra_rows=0)
    check_evict(ctx, c, weights(c, 2), [int(x) for x in c.where], 111 + over, 3, 5)
    c = lh.Cache(43, lens, 16, 2, 64, "bf16", room=0, extra_rows=0)
    check_evict(ctx, c, weights(c, 2), [int(x) for x in c.where], 111 + over, 3, 5, with_kept=False)


def test_a_budget_beyond_the_rows_asks_for_no_more_room_than_they_take():
    import torch
    from paper_2605_16637_amd import binding
    c = cache()
    fresh = binding.Context(0)
    rows = sh.i32(np.resize(c.where, 4000))                     # (all but three of them listed again)
    torch.cuda.synchronize()
    before = torch.cuda.mem_get_info()[0]
    fresh.hx_kv_evict(c.pool, c.seqs, rows, sh.dev(weights(c, 1)), MOST)
    torch.cuda.synchronize()
    assert before - torch.cuda.mem_get_info()[0] < 64 << 20     # 4000 budgets would be 32 TB
    assert lh.status(fresh) == -6
    fresh.close()
