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


def test_a_ragged_life_of_rounds_becomes_the_training_masks():
    """Prompts, steps and rounds that leave rollouts out, by the loop; its kept lists through ngc_replay_visibility, and those into the pass
    over whole sequences: every step's absorbed attention, with the projections applied, is that pass's row of the token."""
    from paper_2604_18002_b200.rollout import NgcLatentRollout
    b = ngc()
    L, B, H, dc, dr, page, cap = 2, 3, 4, 256, 32, 32, 8
    prompt, steps, scale = [70, 33, 130], 80, (128 + dr) ** -0.5
    T = [p + steps for p in prompt]
    rounds_at = {10: [2, -1, 3], 41: [3, 2, -1], 63: [2, 2, 2]}
    latent, rope = [normal((L, n, dc), 500 + i) for i, n in enumerate(T)], [normal((L, n, dr), 520 + i) for i, n in enumerate(T)]
    g = torch.Generator().manual_seed(17)
    U, W = ((torch.randn((L, H, 128, dc), generator=g) / dc ** 0.5).to(bf16) for _ in range(2))
    qn, qr = [normal((L, n, H, 128), 540 + i) for i, n in enumerate(T)], [normal((L, n, H, dr), 560 + i) for i, n in enumerate(T)]
    ro = NgcLatentRollout(L, B, H, dc, dr, n_pages=24, pages_cap=cap, max_new=sum(prompt), scale=scale, page=page, lists=b.LISTS_PER_LAYER)
    ro.update(ints(prompt))
    ro.write(torch.cat([x[:, :p] for x, p in zip(latent, prompt)], 1).cuda(), torch.cat([x[:, :p] for x, p in zip(rope, prompt)], 1).cuda())
    got, n_new = [torch.zeros((L, n, H, 128)) for n in T], ints([1] * B)
    own = [[] for _ in range(B)]                                               # per rollout: (kept, budget, alive before, total before) of its rounds
    for i in range(steps):
        now = [p + i for p in prompt]
        if i in rounds_at:
            lens = host(ro.pool.lens).copy()
            units = -(-lens // page)
            logits = torch.randn((B, L, cap), generator=g)
            for s in range(B):
                for l in range(L):
                    logits[s, l, int(units[s, l]):] = -float("inf")
            ro.evict(logits.cuda(), ints(units.max(1).tolist()), None, ints(rounds_at[i]), 11, i, n_new, n_slots=B)
            for s in range(B):
                if rounds_at[i][s] >= 0:
                    own[s].append((host(ro.kept_sorted)[s], rounds_at[i][s], lens[s], now[s]))
        else:
            ro.update(n_new, B)
        out = torch.zeros((L, B, H, dc), device="cuda")
        q = torch.stack([torch.einsum("lhd,lhdc->lhc", qn[s][:, now[s]].float(), U.float()) for s in range(B)], 1).to(bf16).cuda()
        r = torch.stack([qr[s][:, now[s]] for s in range(B)], 1).cuda()
        rows = [torch.stack([x[s][:, now[s]] for s in range(B)], 1).cuda() for x in (latent, rope)]
        for l in range(L):
            ro.write(*rows, l, l + 1)
            ro.decode(q, r, out, l, l + 1)
        for s in range(B):
            got[s][:, now[s]] = torch.einsum("lhc,lhdc->lhd", out[:, s].cpu(), W.float())
    ro.check_status()
    # the histories; rollouts with fewer rounds get ones behind their end, which keep nothing
    R = max(len(x) for x in own)
    kept, budget = torch.full((R, B, L, cap), -1, dtype=torch.int32), torch.zeros((R, B), dtype=torch.int32)
    alive, total = torch.full((R, B, L), 10 ** 6, dtype=torch.int32), torch.full((R, B), 2 ** 30, dtype=torch.int32)
    assert sorted(len(x) for x in own) == [2, 2, 3]
    for s in range(B):
        for k, (ks, n, before, at) in enumerate(own[s]):
            kept[k, s], budget[k, s], alive[k, s], total[k, s] = torch.as_tensor(ks), n, torch.as_tensor(before), at
        for k in range(len(own[s]), R):
            alive[k, s] = torch.as_tensor(host(ro.pool.lens)[s])
    most = cap * page
    pos, count, st = torch.empty((R, B, L, cap * page), dtype=torch.int32, device="cuda"), torch.empty((R, B, L), dtype=torch.int32, device="cuda"), b.new_status()
    b.ngc_replay_visibility(kept.cuda(), budget.cuda(), alive.cuda(), total.cuda(), page, most, pos, count, status=st)
    assert status_value(st) == 0
    seqs = b.NgcLatentSeqs(torch.tensor([0] + np.cumsum(T).tolist()).cuda(), ints(T), max(T))
    kv = torch.cat([torch.cat([torch.einsum("ltc,lhdc->lthd", x.float(), w.float()).to(bf16) for w in (U, W)], -1) for x in latent], 1).cuda()
    q = torch.cat([torch.cat([a, c], -1) for a, c in zip(qn, qr)], 1).cuda()
    out = torch.zeros((L, sum(T), H, 128), device="cuda")
    ws = b.alloc_workspace(b.latent_replay_workspace_bytes(seqs, q, kv, b.LISTS_PER_LAYER, R))
    b.ngc_latent_replay_attn(seqs, q, kv, torch.cat(rope, 1).cuda(), out, None, pos, count, total.cuda(), lists=b.LISTS_PER_LAYER, ws=ws, status=st)
    assert status_value(st) == 0
    for s in range(B):
        at = sum(T[:s])
        a, c = got[s][:, prompt[s]:], out[:, at + prompt[s]: at + T[s]].cpu()
        # roundings on the way: the absorbed query, keys, values and probabilities, each half a step of bf16 (2**-8); scores are sums of
        # some 300 products of size 1 / 13 with independent roundings, so they move by 0.01 or so, outputs by a few hundredths of their size
        assert float((a - c).norm() / c.norm()) <= 0.02


def test_a_captured_round_follows_its_budgets():
    """Eviction, books and growth in one graph, replayed with other budgets (rollouts left out change), beside the same calls made one by one."""
    from paper_2604_18002_b200.rollout import NgcLatentRollout
    b = ngc()
    L, B, page, cap = 2, 4, 32, 8
    ro = [NgcLatentRollout(L, B, 4, 128, 16, n_pages=40, pages_cap=cap, max_new=600, scale=0.1, page=page, lists=b.LISTS_PER_LAYER) for _ in range(2)]
    n, protect, budget, n_new = ints([0] * B), ints([1] * B), ints([-1] * B), ints([0] * B)
    logits = torch.zeros((B, L, cap), device="cuda")

    def round_of(k):
        ro[k].evict(logits, n, protect, budget, 21, 4, n_new, n_slots=300)
    for k in range(2):
        ro[k].update(ints([160, 90, 33, 250]))
        round_of(k)                                                            # (all left out: nothing happens)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        round_of(0)
    for i, (budgets, new) in enumerate([([3, -1, 1, 5], [1, 100, 1, 0]), ([-1, 2, -1, 2], [70, 1, 64, 3]), ([2, 1, 1, -1], [-1, 5, 0, 90])]):
        n.copy_(ints((-(-host(ro[1].pool.lens) // page)).min(1).tolist()))
        budget.copy_(ints(budgets))
        n_new.copy_(ints(new))
        logits.copy_(torch.randn((B, L, cap), generator=torch.Generator().manual_seed(i)).cuda())
        before = books(ro[1])
        graph.replay()
        round_of(1)
        assert torch.equal(ro[0].kept_sorted, ro[1].kept_sorted)
        want = ora.pool_update(*before, page, np.array(new), 300, host(ro[1].kept_sorted), np.array(budgets))
        assert want[5] == set()
        for k in range(2):
            same_books(ro[k], want, f"round {i}, {'captured' if k == 0 else 'eager'}")
            ro[k].check_status()
