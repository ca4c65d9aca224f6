"""Books of a pool where pages or slots run short: who grows, who does not, and how a caller goes on."""
import numpy as np
import pytest

from oracle import latent as ora
from test_gpu_debug_build import debug_library      # noqa: F401
from test_gpu_latent import host, random_pool, run_update

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("lists", [0, 1])
@pytest.mark.parametrize("n_pages,expect", [(28, [1, 0, 1, 0, 1, 500]), (30, [1, 0, 1, 640, 0, 0])])
def test_a_request_too_large_for_the_pool_does_not_stop_the_others(lists, n_pages, expect):
    """2 + 1 + 1 + 0 + 3 + 2 = 9 pages are in use; wanted are 1, 32, 0, 20, 1 and 15 of the 19 or 21 that are free."""
    pool = random_pool(2, 6, 32, 60, n_pages, [[64], [32], [10], [0], [96], [33]], lists, 3)
    before = host(pool.lens).copy()
    assert run_update(pool, [1, 1000, 1, 640, 1, 500], 4000) == {ora.POOL_FULL}
    assert (host(pool.lens) - before == np.array(expect)[:, None]).all()


@pytest.mark.parametrize("B,seed", [(9, 0), (9, 1), (33, 2), (300, 3), (1000, 4), (8192, 5)])
def test_who_grows_in_a_short_pool(B, seed):
    """Large and small requests in any order, many more of them than pages, on lists with different numbers of free pages."""
    rng = np.random.default_rng(seed)
    page, cap = 32, 40
    lens = rng.integers(0, 200, (B, 3))
    n_pages = int((-(-lens // page)).sum(0).max()) + int(rng.integers(B // 2, 3 * B))
    pool = random_pool(3, B, page, cap, n_pages, lens, 1, seed)
    n_new = np.where(rng.random(B) < 0.3, rng.integers(100, 1000 if B < 5000 else 250, B), rng.integers(-1, 40, B))
    assert run_update(pool, n_new, int(np.maximum(n_new, 0).sum())) == {ora.POOL_FULL}
    live = host(pool.page_table)
    for g in range(3):
        mine = live[:, g][live[:, g] >= 0]
        assert len(set(mine)) == len(mine) == int(host(pool.page_used)[g].sum())


def test_a_sequence_that_grew_on_some_lists_only_can_be_finished_and_admitted_anew():
    page = 32
    pool = random_pool(2, 3, page, 8, 12, [[64, 64], [96, 128], [0, 0]], 1, 5)
    free = (host(pool.page_used) == 0).sum(1)
    assert free.tolist() == [7, 6]
    assert run_update(pool, [0, 0, 7 * page], 7 * page) == {ora.POOL_FULL}                           # fits on the first list only
    assert host(pool.lens)[2].tolist() == [7 * page, 0]
    assert run_update(pool, [1, 0, -1], 4) == set()
    assert host(pool.lens)[2].tolist() == [0, 0]
    assert run_update(pool, [0, 0, 5 * page], 5 * page) == set()
    assert host(pool.lens).tolist() == [[65, 65], [96, 128], [5 * page, 5 * page]]


@pytest.mark.parametrize("n_slots", [60, 5000])
def test_a_sequence_with_more_new_tokens_than_slots_does_not_evict_either(n_slots):
    """It is left as it was, pages and length, in a round too; those behind it that end or only evict are served."""
    page = 32
    pool = random_pool(2, 5, page, 6, 40, [[64, 60], [100, 96], [128, 128], [70, 70], [33, 33]], 1, 6)
    before = [host(x).copy() for x in (pool.page_table, pool.lens)]
    budget = np.array([1, 2, 2, 1, 1])
    kept = np.full((5, 2, 2), -1)
    kept[0, :, 0], kept[1], kept[2], kept[3, :, 0], kept[4, :, 0] = 1, [0, 2], [1, 3], 2, 0
    assert run_update(pool, [20, n_slots, 0, -1, 5], n_slots, kept, budget) == {ora.BAD_COUNTS}
    assert (host(pool.page_table)[1] == before[0][1]).all() and (host(pool.lens)[1] == before[1][1]).all()
    assert host(pool.lens)[[0, 2, 3, 4]].tolist() == [[52, 48], [64, 64], [0, 0], [33, 33]]      # (the last one's 5 tokens have no slots either)


@pytest.mark.parametrize("B,seed", [(33, 2), (300, 3)])
def test_a_short_pool_on_the_bounds_checking_build(B, seed, debug_library):      # noqa: F811
    test_who_grows_in_a_short_pool(B, seed)
    test_a_sequence_with_more_new_tokens_than_slots_does_not_evict_either(60)
