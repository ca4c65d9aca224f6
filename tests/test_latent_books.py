"""The plain books of a page pool where pages or slots run short."""
import numpy as np

from oracle import latent as ora


def state(lens, page, cap, n_pages):
    lens = np.asarray(lens, np.int32)
    B, G = lens.shape
    table, used = np.full((B, G, cap), -1, np.int32), np.zeros((G, n_pages), np.uint8)
    for g in range(G):
        at = 0
        for b in range(B):
            have = -(-int(lens[b, g]) // page)
            table[b, g, :have] = np.arange(at, at + have)
            used[g, at: at + have] = 1
            at += have
    return table, used, lens


def test_a_request_that_does_not_fit_leaves_the_pages_to_those_after_it():
    table, used, lens, slots, first, problems = ora.pool_update(*state([[0], [32]], 32, 120, 11), 32, np.array([3200, 1]), 4000)
    assert problems == {ora.POOL_FULL} and lens.tolist() == [[0], [33]]
    assert (slots[0, :3200] == -1).all() and slots[0, 3200] == 1 * 32 and used.sum() == 2


def test_shortage_is_each_lists_own_and_can_be_undone():
    s = state([[64, 64], [0, 32]], 32, 8, 7)
    table, used, lens, slots, first, problems = ora.pool_update(*s, 32, np.array([0, 160]), 160)
    assert problems == {ora.POOL_FULL} and lens.tolist() == [[64, 64], [160, 32]] and (slots[0] >= 0).all() and (slots[1] == -1).all()
    table, used, lens, slots, first, problems = ora.pool_update(table, used, lens, 32, np.array([0, -1]), 1)
    assert problems == set() and lens.tolist() == [[64, 64], [0, 0]] and used.sum(1).tolist() == [2, 2]


def test_more_new_tokens_than_slots_leave_a_sequence_as_it_was():
    s = state([[64], [64], [40]], 32, 8, 20)
    kept, budget = np.array([[[1]], [[0]], [[1]]]), np.array([1, 1, 1])
    table, used, lens, slots, first, problems = ora.pool_update(*s, 32, np.array([5, 60, -1]), 60, kept, budget)
    assert problems == {ora.BAD_COUNTS} and lens.tolist() == [[37], [64], [0]]
    assert table[1, 0, :3].tolist() == [2, 3, -1] and (slots[0, 5:] == -1).all()
