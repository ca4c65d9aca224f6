"""The plain implementations of oracle/latent.py against what they must satisfy: sets, identities between the two forms,
central differences."""
import numpy as np
import pytest

from oracle import latent as ora


def test_pool_books_conserve_pages():
    rng = np.random.default_rng(0)
    B, G, cap, page, P = 6, 2, 5, 4, 17
    table, used, lens = np.full((B, G, cap), -1, np.int32), np.zeros((G, P), np.uint8), np.zeros((B, G), np.int32)
    for step in range(40):
        n_new = rng.integers(-1, 9, B)
        kept = budget = None
        if step % 3 == 2:
            have = -(-lens // page)
            budget = np.minimum(rng.integers(-1, 3, B), have.min(1))
            kept = np.full((B, G, 3), -1, np.int32)
            for b in range(B):
                for g in range(G):
                    if budget[b] > 0:
                        kept[b, g, : budget[b]] = np.sort(rng.permutation(have[b, g])[: budget[b]])
        before = [x.copy() for x in (table, used, lens)]
        table, used, lens, slots, first, problems = ora.pool_update(table, used, lens, page, n_new, 64, kept, budget)
        assert problems <= {ora.STRIP_FULL, ora.POOL_FULL}
        for g in range(G):
            owned = [int(x) for b in range(B) for x in table[b, g] if x >= 0]
            assert sorted(owned) == sorted(np.flatnonzero(used[g]))                   # every page once, and no others used
            assert all((table[b, g] >= 0).sum() == -(-lens[b, g] // page) for b in range(B))
            given = slots[g][slots[g] >= 0]
            assert len(set(given)) == len(given)
            for b in range(B):
                mine = slots[g, first[b]: first[b + 1]]
                if len(mine) and mine[0] >= 0:                                        # the last places of the sequence, in order
                    pos = np.arange(lens[b, g] - len(mine), lens[b, g])
                    assert np.array_equal(mine, table[b, g, pos // page] * page + pos % page)
        assert before[0].shape == table.shape


def test_absorbed_form_is_the_expanded_form_with_its_projections():
    rng = np.random.default_rng(1)
    T, H, dc, dr, page = 37, 3, 128, 16, 32
    c, r, qn, qr = rng.standard_normal((T, dc)), rng.standard_normal((T, dr)), rng.standard_normal((H, 128)), rng.standard_normal((H, dr))
    U, W = rng.standard_normal((2, H, 128, dc)) / dc ** 0.5
    rows = np.zeros((1, 3, page, dc + dr))
    rows[0, 2], rows[0, 0, :5] = np.concatenate([c, r], -1)[:32], np.concatenate([c, r], -1)[32:]
    ql = np.einsum("hd,hdc->hc", qn, U)
    o, _ = ora.decode(rows, np.array([[[2, 0, -1]]]), np.array([[T]]), ql[None, None], qr[None, None], 0.1, 0)
    absorbed = np.einsum("hc,hdc->hd", o[0, 0], W)
    kv = np.concatenate([np.einsum("tc,hdc->thd", c, U), np.einsum("tc,hdc->thd", c, W)], -1)
    q = np.zeros((T, H, 128 + dr))
    q[-1] = np.concatenate([qn, qr], -1)
    out, lse, _, _ = ora.replay(q, kv, r, ora.visible(T, []), 0.1)
    assert np.abs(out[-1] - absorbed).max() < 1e-12
    z = 0.1 * (ql @ c.T + qr @ r.T)
    assert np.allclose(lse[:, -1], np.log(np.exp(z).sum(-1)))


def test_visibility_is_the_cache_as_it_was():
    see = ora.visible(8, [(3, [0, 2]), (6, [2, 5]), (20, [])])
    assert see[2].tolist() == [1, 1, 1, 0, 0, 0, 0, 0] and see[3].tolist() == [1, 0, 1, 1, 0, 0, 0, 0]
    assert see[5].tolist() == [1, 0, 1, 1, 1, 1, 0, 0] and see[7].tolist() == [0, 0, 1, 0, 0, 1, 1, 1]


def test_gradient_by_the_formula_is_the_difference_quotient():
    rng = np.random.default_rng(2)
    T, H, dr = 13, 2, 16
    x = [rng.standard_normal(s) for s in ((T, H, 128 + dr), (T, H, 256), (T, dr))]
    see, scale, go = ora.visible(T, [(4, [1, 3]), (9, [3, 5, 8])]), 0.11, rng.standard_normal((T, H, 128))
    out, lse, _, _ = ora.replay(*x, see, scale)
    grads = [g for g, _ in ora.replay_grad(*x, see, scale, out, lse, go)]
    for k in range(3):
        for _ in range(4):
            d = rng.standard_normal(x[k].shape)
            y = [[t + (s * 1e-5 * d if i == k else 0) for i, t in enumerate(x)] for s in (1, -1)]
            numeric = sum(s * (ora.replay(*v, see, scale)[0] * go).sum() for s, v in zip((1, -1), y)) / 2e-5
            assert abs(numeric - (grads[k] * d).sum()) < 1e-6 * max(1.0, abs(numeric))


def test_a_query_that_sees_nothing_is_zero():
    rng = np.random.default_rng(3)
    see = ora.visible(3, [])
    see[1] = False
    x = [rng.standard_normal(s) for s in ((3, 1, 144), (3, 1, 256), (3, 16))]
    out, lse, ob, _ = ora.replay(*x, see, 0.1)
    assert (out[1] == 0).all() and lse[0, 1] == -np.inf and np.isfinite(ob).all()
    grads = ora.replay_grad(*x, see, 0.1, out, lse, rng.standard_normal((3, 1, 128)))
    assert all(np.isfinite(g).all() and np.isfinite(b).all() for g, b in grads) and (grads[0][0][1] == 0).all()
