"""Latent-attention calls at their edges: the bounds-checking build, what a call must not touch, calls at once, captured calls,
rows beyond 4 GB, many units, results that must not depend on chance, numbers at the edge of the range."""
import numpy as np
import pytest
import torch

import test_gpu_latent as t_lat
from helpers import ngc, status_value
from oracle import latent as ora
from test_gpu_debug_build import debug_library      # noqa: F401
from test_gpu_latent import Replay, assert_within, bf16, device_history, f32, history, host, normal, random_pool, run_decode, run_update

pytestmark = pytest.mark.gpu

CASES = [(t_lat.test_pool_books_follow_a_life_of_steps_rounds_and_ends, (3, 1, 5, 32, 1)),
         (t_lat.test_pool_books_follow_a_life_of_steps_rounds_and_ends, (2, 2, 40, 64, 2)),
         (t_lat.test_pool_problems_leave_their_sequence_alone, ("full",)), (t_lat.test_pool_problems_leave_their_sequence_alone, ("kept",)),
         (t_lat.test_rows_land_in_their_slots_and_nowhere_else, (3, 1, 128, 16, 32, 77, (1, 3)))] + [
        (t_lat.test_decode_matches_the_definition, (i,)) for i in (2, 3, 6, 8, 10)] + [
        (t_lat.test_replay_matches_the_definition, (i, bf16)) for i in (1, 2, 4, 7)] + [(t_lat.test_gradient_matches_the_formula, (i,)) for i in (1, 2, 4, 7)]


@pytest.mark.parametrize("i", range(len(CASES)), ids=[f"{f.__name__}-{i}" for i, (f, _) in enumerate(CASES)])
def test_small_latent_case_on_the_bounds_checking_build(i, debug_library):      # noqa: F811
    fn, args = CASES[i]
    fn(*args)


# ------------------------------------------------------------------ what is not touched

def behind(n, dtype, fill):
    """A tensor of n elements and the whole allocation with 1024 more of them behind it."""
    whole = torch.full((n + 1024,), fill, dtype=dtype, device="cuda")
    return whole[:n], whole[n:]


@pytest.mark.parametrize("H,lens", [(5, [130, 0, 64]), (40, [700, 5, 1]), (128, [333, 2000, 64])])
def test_decode_writes_its_outputs_and_workspace_and_nothing_else(H, lens):
    b = ngc()
    pool = random_pool(1, 3, 32, 64, 100, lens, 0, 3, 256, 32)
    books = [x.clone() for x in (pool.rows, pool.page_table, pool.page_used, pool.lens)]
    out, out_tail = behind(3 * H * 256, f32, 7.0)
    need = b.latent_decode_workspace_bytes(pool, H)
    ws, ws_tail = behind(need, torch.uint8, 0xAB)
    ql, qr, st = normal((1, 3, H, 256), 1), normal((1, 3, H, 32), 2), b.new_status()
    b.ngc_latent_decode(pool, ql.cuda(), qr.cuda(), out.view(1, 3, H, 256), 0.08, ws=ws, status=st)
    want, bound = ora.decode(*[host(x) for x in (books[0], books[1], books[3])], host(ql), host(qr), 0.08, 0)
    assert_within(out.view(1, 3, H, 256), want, bound)
    assert status_value(st) == 0 and bool((out_tail == 7).all()) and bool((ws_tail == 0xAB).all())
    for x, y in zip(books, (pool.rows, pool.page_table, pool.page_used, pool.lens)):
        assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))


def test_replay_and_gradient_stay_in_their_workspace():
    b = ngc()
    r = Replay(1, 2, 2, 48, [200, 130], 3, 5, [(0.4, 0.5), (0.8, 0.5)])
    for back in (False, True):
        need = b.latent_replay_workspace_bytes(r.seqs, r.dev[0], r.dev[1], 0, 2, back)
        ws, tail = behind(need, torch.uint8, 0xAB)
        r.ws = lambda backward, ws=ws: ws
        (r.backward if back else r.forward)()
        assert bool((tail == 0xAB).all()) and status_value(r.st) == 0
    r.check_forward()
    r.check_backward()


# ------------------------------------------------------------------ at once, captured, repeated

def test_two_decodes_and_two_gradients_at_once():
    b = ngc()
    pools = [random_pool(1, 20, 64, 40, 900, np.random.default_rng(s).integers(0, 2500, 20), 0, s, 512, 64) for s in (1, 2)]
    qs = [(normal((1, 20, 16, 512), s).cuda(), normal((1, 20, 16, 64), s + 9).cuda()) for s in (1, 2)]
    wss = [b.alloc_workspace(b.latent_decode_workspace_bytes(p, 16)) for p in pools]
    reps = [Replay(1, 2, 4, 64, [700, 300 + 50 * s], 0, 30 + s, [(0.4, 0.5)]) for s in (0, 1)]
    for r in reps:
        r.forward()
    want = []
    for p, q, w in zip(pools, qs, wss):
        o = torch.zeros((1, 20, 16, 512), dtype=bf16, device="cuda")
        b.ngc_latent_decode(p, *q, o, 0.07, ws=w)
        want.append(o)
    grads = [[g.clone() for g in r.backward()] for r in reps]
    spaces = [r.ws(True) for r in reps]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(5):
        got = [torch.zeros_like(w) for w in want]
        outs = [[torch.full_like(g, 7) for g in gs] for gs in grads]
        torch.cuda.synchronize()
        for k, s in enumerate(streams):
            with torch.cuda.stream(s):
                b.ngc_latent_decode(pools[k], *qs[k], got[k], 0.07, ws=wss[k])
                r = reps[k]
                b.ngc_latent_replay_attn_backward(r.seqs, *r.dev[:3], r.out, r.lse, r.dev[3], *outs[k], *r.alive, lists=0, ws=spaces[k])
                b.ngc_latent_decode(pools[k], *qs[k], got[k], 0.07, ws=wss[k])
        torch.cuda.synchronize()
        assert all(torch.equal(a, w) for a, w in zip(got, want))
        assert all(torch.equal(a[n], g[n]) for a, g in zip(outs, grads) for n in range(3))


def test_a_captured_step_follows_its_inputs():
    """Books, rows and decode of a step in one graph, replayed with other counts, rows and queries; padding slots stay unused."""
    b = ngc()
    L, B, H, dc, dr, page, cap = 2, 4, 8, 256, 32, 32, 6
    from paper_2604_18002_b200.rollout import NgcLatentRollout
    ro = [NgcLatentRollout(L, B, H, dc, dr, 40, cap, 64, 0.07, page, lists=b.LISTS_PER_LAYER) for _ in range(2)]
    for r in ro:
        r.pool.rows.zero_()
    n_new = torch.zeros(B, dtype=torch.int32, device="cuda")
    lat, rope = torch.zeros((L, 64, dc), dtype=bf16, device="cuda"), torch.zeros((L, 64, dr), dtype=bf16, device="cuda")
    ql, qr = torch.zeros((L, B, H, dc), dtype=bf16, device="cuda"), torch.zeros((L, B, H, dr), dtype=bf16, device="cuda")
    outs = [torch.zeros((L, B, H, dc), device="cuda") for _ in range(2)]

    def step(k):
        ro[k].update(n_new)
        ro[k].write(lat, rope)
        ro[k].decode(ql, qr, outs[k])
    step(0)                                                       # (no tokens: configures the kernels)
    step(1)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(0)
    # (a capture runs nothing)
    for i, counts in enumerate([[5, 0, 16, 3], [1, 1, 1, 1], [20, 0, 1, 1], [1, 30, -1, 2], [2, 1, 7, 1]]):
        n_new.copy_(torch.tensor(counts, dtype=torch.int32))
        for t, s in ((lat, 1), (rope, 2), (ql, 3), (qr, 4)):
            t.copy_(normal(t.shape, 50 * i + s).cuda())
        graph.replay()
        step(1)
        torch.cuda.synchronize()
        for x in ("page_table", "page_used", "lens"):
            assert torch.equal(getattr(ro[0].pool, x), getattr(ro[1].pool, x)), (i, x)
        assert torch.equal(ro[0].slots, ro[1].slots) and torch.equal(outs[0], outs[1])
        want, bound = ora.decode(*[host(x) for x in (ro[0].pool.rows, ro[0].pool.page_table, ro[0].pool.lens)], host(ql), host(qr), 0.07, 1)
        assert_within(outs[0], want, bound, f"step {i}")
    for r in ro:
        r.check_status()


def test_a_captured_gradient_follows_its_inputs():
    r = Replay(1, 2, 2, 64, [300, 170], 0, 70, [(0.3, 0.5), (0.7, 0.5)])
    b = ngc()
    r.forward()
    r.backward()
    torch.cuda.synchronize()
    ws = [r.ws(False), r.ws(True)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        b.ngc_latent_replay_attn(r.seqs, *r.dev[:3], r.out, r.lse, *r.alive, lists=0, ws=ws[0], status=r.st)
        b.ngc_latent_replay_attn_backward(r.seqs, *r.dev[:3], r.out, r.lse, r.dev[3], *r.grads, *r.alive, lists=0, ws=ws[1], status=r.st)
    for s in (1, 2):
        for name, t in zip(("q", "kv", "kr", "go"), r.dev):
            setattr(r, name, normal(t.shape, 90 + 7 * s + len(name)))
            t.copy_(getattr(r, name).cuda())
        graph.replay()
        torch.cuda.synchronize()
        r.check_forward()
        r.check_backward()
    assert status_value(r.st) == 0


def test_the_same_bits_in_every_run():
    r = Replay(2, 3, 5, 64, [513, 900, 64], 2, 75, [(0.2, 0.5), (0.6, 0.4)], 1, 16)
    pool = random_pool(2, 9, 32, 100, 950, np.random.default_rng(3).integers(1, 3000, (9, 2)), 1, 6, 384, 48)
    first = None
    for _ in range(4):
        r.forward()
        got = [r.out, r.lse] + r.backward() + [run_decode(pool, 20, 0.08)[2]]
        got = [x.clone().view(torch.uint8) for x in got]
        first = first or got
        assert all(torch.equal(a, c) for a, c in zip(got, first))


# ------------------------------------------------------------------ sizes

def test_pool_of_more_than_four_gigabytes():
    b = ngc()
    P, page, dc, dr = 60000, 64, 512, 64                          # 4.4 GB in one layer
    pool = b.new_latent_pool(1, 2, dc, dr, P, 8, page)
    pool.page_used[0, : P - 9] = 1                                # the last pages are the free ones
    slots, first, st = torch.empty((1, 500), dtype=torch.int32, device="cuda"), torch.empty(3, dtype=torch.int32, device="cuda"), b.new_status()
    b.ngc_pool_update(pool, torch.tensor([300, 200], dtype=torch.int32).cuda(), slots, first, status=st)
    assert int(slots[0, 0]) == (P - 9) * page and int(slots[0, -1]) == (P - 1) * page + 7
    lat, rope = normal((1, 500, dc), 1), normal((1, 500, dr), 2)
    b.ngc_latent_write(pool, slots, lat.cuda(), rope.cuda(), status=st)
    ql, qr, out, st2 = run_decode(pool, 16, 0.07)
    assert status_value(st) == 0 and status_value(st2) == 0
    rows = torch.cat([lat, rope], -1)[0].float().numpy()
    few = np.zeros((1, 9, page, dc + dr), np.float32)             # the last nine pages
    few[0, :5].reshape(-1, dc + dr)[:300], few[0, 5:].reshape(-1, dc + dr)[:200] = rows[:300], rows[300:]
    table = np.array([[[0, 1, 2, 3, 4, -1, -1, -1]], [[5, 6, 7, 8, -1, -1, -1, -1]]])
    want, bound = ora.decode(few, table, np.array([[300], [200]]), host(ql), host(qr), 0.07, 0)
    assert_within(out, want, bound)


def test_decode_of_more_units_than_threads():
    rng = np.random.default_rng(4)
    lens = rng.integers(0, 70, (500, 2))
    lens[rng.random((500, 2)) < 0.3] = 0
    pool = random_pool(2, 500, 32, 3, 1700, lens, 1, 8, 128, 32)
    ql, qr, out, st = run_decode(pool, 9, 0.08)
    want, bound = ora.decode(host(pool.rows), host(pool.page_table), host(pool.lens), host(ql), host(qr), 0.08, 1)
    assert status_value(st) == 0
    assert_within(out, want, bound)


@pytest.mark.parametrize("H,dc,lens", [(16, 512, [64 * 11]), (5, 128, [64 * 12]), (17, 384, [64 * 13 - 1, 0]), (3, 256, [64 * 148 + 5]), (16, 512, [20001, 3, 0, 5000]),
                                       (128, 512, [4000, 1, 700, 2600]), (64, 128, [9000, 9000, 30, 9000, 64])])
def test_decode_of_sequences_in_few_and_in_many_parts(H, dc, lens):
    pool = random_pool(1, len(lens), 64, -(-max(lens) // 64), sum(-(-n // 64) for n in lens) + 1, lens, 0, 31, dc, 64)
    for out_dtype in (bf16, f32):
        ql, qr, out, st = run_decode(pool, H, 0.1, out_dtype)
        want, bound = ora.decode(host(pool.rows), host(pool.page_table), host(pool.lens), host(ql), host(qr), 0.1, 0, out_dtype is bf16)
        assert status_value(st) == 0
        assert_within(out, want, bound)


@pytest.mark.parametrize("seed", range(8))
def test_decode_of_random_shapes(seed):
    rng = np.random.default_rng(100 + seed)
    L, B, H = int(rng.integers(1, 4)), int(rng.integers(1, 9)), int(rng.integers(1, 129))
    dc, dr, page, lists = int(rng.choice([128, 256, 384, 512])), int(rng.choice([16, 32, 48, 64])), int(rng.choice([32, 64])), int(rng.integers(0, 3))
    lens = rng.integers(0, int(rng.choice([3, 70, 900])), (B, L if lists else 1))
    cap = max(1, -(-int(lens.max()) // page))
    pool = random_pool(L, B, page, cap, int((-(-lens // page)).sum(0).max()) + 1, lens, lists, seed, dc, dr)
    scale = float(rng.uniform(0.02, 0.3))
    ql, qr, out, st = run_decode(pool, H, scale, bf16 if seed % 2 else f32)
    want, bound = ora.decode(host(pool.rows), host(pool.page_table), host(pool.lens), host(ql), host(qr), scale, lists, bool(seed % 2))
    assert status_value(st) == 0
    assert_within(out, want, bound)


@pytest.mark.parametrize("seed", range(6))
def test_replay_of_random_shapes(seed):
    rng = np.random.default_rng(200 + seed)
    L, B, H, dr = int(rng.integers(1, 3)), int(rng.integers(1, 6)), int(rng.integers(1, 5)), int(rng.choice([16, 32, 48, 64]))
    lens = [int(x) for x in rng.integers(0, int(rng.choice([5, 150, 600])), B)]
    lens[0] += 1
    rounds = None if seed % 3 == 0 else [(f, float(rng.uniform(0, 1))) for f in np.sort(rng.uniform(0.05, 1, int(rng.integers(1, 6))))]
    r = Replay(L, B, H, dr, lens, int(rng.integers(0, 3)), 300 + seed, rounds, int(rng.integers(0, 3)), int(rng.choice([1, 4, 32])))
    r.forward(f32 if seed % 2 else bf16)
    r.backward()
    assert status_value(r.st) == 0
    r.check_forward()
    r.check_backward()


@pytest.mark.parametrize("seed", range(3))
def test_histories_that_leave_halves_of_tiles(seed):
    """Rounds that keep or drop 64 keys at a time, at moments inside a block of queries: tiles of which only the first half is left,
    only the second, a few keys of one, none; more items than SMs."""
    rng = np.random.default_rng(400 + seed)
    lens, H = [1400, 1337, 1281, 1410], 8
    r = Replay(1, len(lens), H, 64, lens, 1, 410 + seed, [(0.5, 0.5)])
    r.hist = []
    for n in lens:
        alive, at, rounds = np.zeros(0, np.int64), 0, []
        for fired in (655, 700 + 7 * seed, 1024, 1279):
            alive = np.concatenate([alive, np.arange(at, fired)])
            at = fired
            share = rng.choice([0.0, 0.0, 1.0, 1.0, 0.05], fired // 64 + 1)           # of every 64 keys
            alive = alive[rng.random(len(alive)) < share[alive // 64]]
            rounds.append((fired, alive))
        r.hist.append([rounds])
    r.alive = device_history(r.hist, len(lens), 1)
    r.forward(f32 if seed % 2 else bf16)
    r.backward()
    assert status_value(r.st) == 0
    r.check_forward()
    r.check_backward()


def test_long_histories_and_sequences_beyond_the_plans_masks():
    """More than 256 tiles of keys (the masks that are planned ahead), nearly all of which have gone."""
    T = 33500
    r = Replay(1, 1, 1, 16, [T], 0, 81, [(0.5, 0.001), (0.9, 0.5)])
    r.forward(f32)
    r.backward()
    assert status_value(r.st) == 0
    # the last 300 queries by the definition; their keys' gradients too, since no earlier query sees tokens 33200 on
    see = np.zeros((300, T), bool)
    alive = [x for x in r.hist[0][0][-1][1]]
    for i in range(300):
        see[i, alive] = True
        see[i, r.hist[0][0][-1][0]: T - 300 + i + 1] = True
    q, kv, kr, go = (host(x[0]).astype(np.float64) for x in (r.q, r.kv, r.kr, r.go))
    k = np.concatenate([kv[:, 0, :128], kr], -1)
    z = np.where(see, r.scale * q[-300:, 0] @ k.T, -np.inf)
    p = np.exp(z - z.max(-1, keepdims=True))
    p /= p.sum(-1, keepdims=True)
    want = p @ kv[:, 0, 128:]
    e = 2 * (144 * ora.U32 * r.scale * (np.abs(q[-300:, 0]) @ np.abs(k).T).max(-1, keepdims=True)) + ora.EXP + T * ora.U32
    assert_within(r.out[0, -300:, 0], want, (ora.U16 + e) * (p @ np.abs(kv[:, 0, 128:])) + e * np.abs(want))
    grad_v = (p.T @ go[-300:, 0])[-300:]
    assert_within(r.grads[1][0, -300:, 0, 128:], grad_v, (ora.U16 + 2 * e.max()) * (p.T @ np.abs(go[-300:, 0]))[-300:] + ora.U16 * np.abs(grad_v))


def test_eviction_of_rows_longer_than_a_warps_buffer():
    rng = np.random.default_rng(5)
    B, cap, page = 3, 1100, 32
    pool = random_pool(2, B, page, cap, 2500, [[1000 * 32 - 5, 700 * 32], [513 * 32, 512 * 32 - 1], [40, 31]], 1, 9)
    have = -(-host(pool.lens) // page)
    budget = np.array([600, 200, 1])
    kept = np.full((B, 2, 600), -1, np.int32)
    for s in range(B):
        for g in range(2):
            last = [have[s, g] - 1] if (s, g) == (0, 0) else []              # a short last page stays last
            kept[s, g, : budget[s]] = np.sort(list(rng.permutation(max(have[s, g] - 1, 1))[: budget[s] - len(last)]) + last)
    assert run_update(pool, [1, 40, 3], 50, kept, budget) == set()


@pytest.mark.parametrize("n_new,n_slots", [([3000, 0, 2500, 1, 900, 64], 6465), ([3000, 0, 9000, 1, 900, 64], 13000), ([5, 5, 5, 5, 5, 4000], 20001), ([1, 2, 4, 5, 6, 7], 9000)])
def test_slots_of_many_tokens_with_sequences_that_do_not_grow(n_new, n_slots):
    pool = random_pool(2, 6, 32, 150, 260, [[100, 90], [64, 64], [10, 33], [0, 0], [96, 90], [33, 33]], 1, 12)
    run_update(pool, n_new, n_slots)
    assert run_update(pool, [1, -1, -1, 200, 0, 3000], n_slots) <= {ora.POOL_FULL, ora.STRIP_FULL}


@pytest.mark.parametrize("n_slots", [40, 9000])
def test_counts_whose_sum_passes_32_bits_get_no_slots(n_slots):
    big = 2 ** 31 - 1
    for n_new in ([big, big, 5, 3, 0, 7], [4, big, big, 5, 3, -1], [2 ** 30, 2 ** 30, 2 ** 30, 2 ** 30, 5, 3], [big] * 6):
        pool = random_pool(2, 6, 32, 8, 60, [[50, 40], [64, 64], [10, 33], [0, 0], [96, 90], [33, 33]], 1, 7)
        assert run_update(pool, n_new, n_slots) <= {ora.BAD_COUNTS}
    B = 700                                                                    # more than a pass over the sequences takes
    pool = random_pool(2, B, 32, 2, 1500, np.full((B, 2), 20), 1, 8)
    n_new = np.ones(B, np.int64)
    n_new[100:400] = big
    assert run_update(pool, n_new, n_slots) == {ora.BAD_COUNTS}


# ------------------------------------------------------------------ numbers

def test_nan_and_infinities_in_alive_rows_stay_with_their_sequence_and_heads():
    pool = random_pool(1, 4, 32, 8, 40, [200, 200, 200, 200], 0, 15, 128, 16)
    clean = host(pool.rows)
    table = host(pool.page_table)
    pool.rows[0, table[1, 0, 3], 5, 7] = float("nan")
    pool.rows[0, table[2, 0, 0], 1, 130] = float("inf")                        # a rotary channel: the score is +-inf
    ql, qr, out, st = run_decode(pool, 6, 0.1)
    want, bound = ora.decode(clean, table, host(pool.lens), host(ql), host(qr), 0.1, 0)
    for s in (0, 3):
        assert_within(out[:, s], want[:, s], bound[:, s])
    assert bool(torch.isnan(out[0, 1]).all())
    up = qr[0, 2, :, 130 - 128].float() > 0                                    # +inf: the row sees an infinite score; -inf: it does not see the key
    assert bool(torch.isnan(out[0, 2, up.cuda()]).all()) and bool(torch.isfinite(out[0, 2, (~up).cuda()]).all())


def test_huge_scores_pick_the_largest():
    pool = random_pool(1, 1, 64, 4, 6, [200], 0, 16, 128, 16)
    ql, qr, out, st = run_decode(pool, 16, 1e4)
    x = host(pool.rows)[0, host(pool.page_table)[0, 0]].reshape(-1, 144)[:200].astype(np.float64)
    z = np.concatenate([host(ql)[0, 0], host(qr)[0, 0]], -1).astype(np.float64) @ x.T
    best = x[z.argmax(-1), :128]
    gap = np.sort(z, -1)[:, -1] - np.sort(z, -1)[:, -2]
    sure = gap * 1e4 > 60                                                      # the second has no weight in fp32
    assert sure.any() and np.abs(host(out)[0, 0][sure] - best[sure]).max() <= 2.0 ** -8 * np.abs(best).max()
