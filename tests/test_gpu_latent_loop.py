"""The rollout loop over a common pool as a serving program runs it: rounds that leave some rollouts out."""
import numpy as np
import pytest
import torch

from helpers import ngc, status_value
from oracle import latent as ora
from test_gpu_latent import bf16, host, normal

pytestmark = pytest.mark.gpu


def books(ro):
    return [host(x).copy() for x in (ro.pool.page_table, ro.pool.page_used, ro.pool.lens)]


def same_books(ro, want, what=""):
    for name, got, w in zip(("table", "used", "lens", "slots", "first"), books(ro) + [host(ro.slots), host(ro.first)], want):
        assert np.array_equal(got, w), f"{what} {name}"


def ints(x):
    return torch.tensor(x, dtype=torch.int32).cuda()


@pytest.mark.parametrize("lists,greedy,protect", [(0, 0, None), (1, 0, None), (1, 1, [1, 1, 9, 1, 0]), (1, 0, [2, 1, 0, 1, 1])])
def test_a_round_leaves_out_rollouts_whose_budget_is_none(lists, greedy, protect):
    """budget -1: the rollout keeps all it has and takes no part in the draw, whatever its counts and logits hold.  On some layers it is a
    page short of the others, so no budget of whole pages would say the same."""
    from paper_2604_18002_b200.rollout import NgcLatentRollout
    b = ngc()
    L, B, page, cap = 2, 5, 32, 8
    G = L if lists else 1
    ro = NgcLatentRollout(L, B, 4, 128, 16, n_pages=60, pages_cap=cap, max_new=700, scale=0.1, page=page, lists=lists)
    ro.update(ints([100, 170, 40, 33, 64]))
    # a first round in which every rollout's second list loses its short last page, the first one's stays
    have = -(-host(ro.pool.lens) // page)
    logits = torch.zeros((B, G, cap))
    for s in range(B):
        logits[s, 0, have[s, 0] - 1] = 50.0
        if lists:
            logits[s, 1, have[s, 1] - 1] = -50.0
    ro.evict(logits.cuda(), ints(have[:, 0].tolist()), None, ints((have[:, 0] - 1).clip(min=1).tolist()), 3, 0, ints([0] * B), greedy=1)
    ro.check_status()
    # now two draw, one is left out with garbage for counts and logits, one is finished, one only grows
    before, page_counts = books(ro), -(-host(ro.pool.lens) // page)
    n, budget, n_new = page_counts.max(1).tolist(), [2, 3, -1, -1, -1], [1, 40, 70, -1, 1]
    n[2] = 77                                                                # (no count of a list of eight)
    logits = torch.randn((B, G, cap), generator=torch.Generator().manual_seed(5))
    logits[2] = float("nan")
    for s in range(2):
        for g in range(G):
            logits[s, g, int(page_counts[s, g]):] = -float("inf")
    logits, prot = logits.cuda(), None if protect is None else ints(protect)
    ro.evict(logits, ints(n), prot, ints(budget), 11, 1, ints(n_new), greedy=greedy)
    assert status_value(ro.status) == 0
    kept = host(ro.kept_sorted)
    assert (kept[2:] == -1).all() and (host(ro.kept_order)[2:] == -1).all()
    want = ora.pool_update(*before, page, np.array(n_new), ro.slots.shape[1], kept, np.array(budget))
    assert want[5] == set()
    same_books(ro, want)
    # the two that draw get what they get alone, and the draw's log-probability goes by the counts of the draw
    assert [host(x).tolist() for x in ro.counts if x is not None][0][:2] == n[:2] and host(ro.counts[2]).tolist() == [2, 3, 0, 0, 0]
    logp, st = torch.full((1, B, G), 7.0, dtype=torch.float64, device="cuda"), b.new_status()
    safe = torch.where(torch.isnan(logits), 0.0, logits)[None]
    b.ngc_evict_logprob(safe, *ro.counts, ro.kept_order, logp, status=st)
    assert status_value(st) == 0 and bool((logp[0, 2:] == 0).all()) and bool(torch.isfinite(logp[0, :2]).all())
    alone = torch.full_like(ro.kept_order[:2], -7)
    order = torch.full_like(alone, -7)
    b.ngc_sample_evict(logits[:2].contiguous(), ints(n[:2]), None if prot is None else prot[:2].contiguous(), ints(budget[:2]), 11, 1, order, alone, None,
                       greedy=greedy, ws=ro.ws_sample, status=st)
    assert torch.equal(alone, ro.kept_sorted[:2]) and torch.equal(order, ro.kept_order[:2]) and status_value(st) == 0


def test_a_budget_below_minus_one_is_reported():
    from paper_2604_18002_b200.rollout import NgcLatentRollout
    ro = NgcLatentRollout(1, 2, 4, 128, 16, n_pages=20, pages_cap=4, max_new=200, scale=0.1, page=32)
    ro.update(ints([70, 70]))
    before = books(ro)
    ro.evict(torch.zeros((2, 1, 4), device="cuda"), ints([3, 3]), None, ints([-2, 1]), 1, 0, ints([0, 0]))
    assert status_value(ro.status) == 1
    want = ora.pool_update(*before, 32, np.array([0, 0]), ro.slots.shape[1], host(ro.kept_sorted), np.array([-2, 1]))
    same_books(ro, want)
