"""Latent attention on the GPU against plain implementations in 64 bits: the pool's books and rows bit for bit, attention and
gradients within bounds that count roundings (see oracle/latent.py)."""
import numpy as np
import pytest
import torch

from helpers import ngc, status_value
from oracle import latent as ora

pytestmark = pytest.mark.gpu

bf16, f32 = torch.bfloat16, torch.float32


def normal(shape, seed, loud=0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(shape, generator=g)
    if loud:
        x[..., :loud] *= 4
    return x.to(bf16)


def host(t):
    return t.detach().cpu().float().numpy() if t.is_floating_point() else t.detach().cpu().numpy()


def assert_within(got, want, bound, what=""):
    got = host(got).astype(np.float64)
    with np.errstate(invalid="ignore"):
        off = np.abs(got - want) / (bound + 1e-30)
        off = np.where((got == want) | (np.abs(got - want) <= 1e-12), 0.0, off)
    assert np.isfinite(got[np.isfinite(want)]).all(), what
    assert off.max() <= 1.0, f"{what}: {off.max():.3g} times the bound at {np.unravel_index(off.argmax(), off.shape)}"


# ------------------------------------------------------------------ books of the pool

def random_pool(L, B, page, cap, n_pages, lens, lists, seed, dc=128, dr=16):
    """A pool in use: every sequence's pages anywhere."""
    b = ngc()
    G = L if lists else 1
    rng = np.random.default_rng(seed)
    lens = np.asarray(lens, np.int32).reshape(B, -1) + np.zeros((B, G), np.int32)
    table, used = np.full((B, G, cap), -1, np.int32), np.zeros((G, n_pages), np.uint8)
    for g in range(G):
        order, at = rng.permutation(n_pages), 0
        for s in range(B):
            have = -(-int(lens[s, g]) // page)
            table[s, g, :have] = order[at: at + have]
            used[g, order[at: at + have]] = 1
            at += have
    rows = normal((L, n_pages, page, dc + dr), seed + 1, 4).cuda()
    return b.NgcLatentPool(rows, torch.as_tensor(table).cuda(), torch.as_tensor(used).cuda(), torch.as_tensor(lens).cuda(), dc, lists)


def run_update(pool, n_new, n_slots, kept=None, budget=None):
    """One call beside the oracle; every book, the slots and the numbers of the tokens are the same.  Returns the problems."""
    b = ngc()
    page = pool.rows.shape[2]
    before = [host(x) for x in (pool.page_table, pool.page_used, pool.lens)]
    n_new = np.asarray(n_new, np.int32)
    G = before[1].shape[0]
    slots = torch.full((G, n_slots), -7, dtype=torch.int32, device="cuda")
    first = torch.full((len(n_new) + 1,), -7, dtype=torch.int32, device="cuda")
    st = b.new_status()
    dev = [None if x is None else torch.as_tensor(np.asarray(x, np.int32)).cuda() for x in (n_new, kept, budget)]
    b.ngc_pool_update(pool, dev[0], slots, first, kept_sorted=dev[1], budget=dev[2], status=st)
    want = ora.pool_update(*before, page, n_new, n_slots, kept, budget)
    for name, got, w in zip(("table", "used", "lens", "slots", "first"), (pool.page_table, pool.page_used, pool.lens, slots, first), want):
        assert np.array_equal(host(got), w), name
    assert (status_value(st) == 0) if not want[5] else (status_value(st) in want[5])
    return want[5]


@pytest.mark.parametrize("L,lists,B,page,seed", [(1, 0, 1, 64, 0), (3, 1, 5, 32, 1), (2, 2, 40, 64, 2), (4, 0, 70, 32, 3)])
def test_pool_books_follow_a_life_of_steps_rounds_and_ends(L, lists, B, page, seed):
    rng = np.random.default_rng(seed)
    cap, G = 9, L if lists else 1
    pool = random_pool(L, B, page, cap, B * cap + 5, np.zeros(B), lists, seed)
    for step in range(12):
        have = -(-host(pool.lens) // page)
        kind = step % 4
        n_new = rng.integers(0, 3 * page if kind == 0 else 2, B)
        n_new = np.minimum(n_new, (cap - 1) * page - host(pool.lens).max(1)).clip(min=0)
        kept = budget = None
        if kind == 2:
            n_new[rng.random(B) < 0.3] = -1
        if kind == 3:
            budget = np.minimum(rng.integers(-1, 5, B), have.min(1)).astype(np.int32)
            k_max = max(1, int(budget.max()))
            kept = np.full((B, G, k_max), -1, np.int32)
            for s in range(B):
                for g in range(G):
                    if budget[s] > 0:
                        kept[s, g, : budget[s]] = np.sort(rng.permutation(have[s, g])[: budget[s]])
        total = int(np.maximum(n_new, 0).sum())
        assert run_update(pool, n_new, total + (3 if step % 2 else max(1, total) - total), kept, budget) == set()
        live = host(pool.page_table)
        for g in range(G):                                     # every page serves one sequence or none
            mine = live[:, g][live[:, g] >= 0]
            assert len(set(mine)) == len(mine) == int(host(pool.page_used)[g].sum())


def test_pool_large_lists_take_several_passes_over_the_map():
    rng = np.random.default_rng(9)
    B, page, n_pages = 1500, 32, 40003                          # more sequences than threads, pages than a pass looks at, odd rows
    lens = rng.integers(0, 700, (B, 2))
    pool = random_pool(2, B, page, 30, n_pages, lens, 1, 4)
    n_new = rng.integers(0, 100, B)
    n_new[::7] = -1
    assert run_update(pool, n_new, int(np.maximum(n_new, 0).sum())) == set()


@pytest.mark.parametrize("what", ["full", "strip", "counts", "kept", "page", "slots", "page_of_growth", "left"])
def test_pool_problems_leave_their_sequence_alone(what):
    page, cap, B = 32, 4, 6
    pool = random_pool(2, B, page, cap, 24 if what != "full" else 17, [[50, 40], [64, 64], [10, 33], [0, 0], [96, 90], [33, 33]], 1, 7)
    n_new, n_slots, kept, budget, expect = np.array([5, 1, 2, 40, 3, 1]), 200, None, None, set()
    if what == "full":
        n_new, expect = np.array([5, 1, 60, 100, 3, 64]), {ora.POOL_FULL, ora.BAD_COUNTS}      # (the last one's 64 are more than 200 slots hold)
    if what == "strip":
        n_new, expect = np.array([5, 1, 2, 129, 33, 1]), {ora.STRIP_FULL}
    if what == "counts":
        pool.lens[1, 0], pool.lens[2, 1], n_new[5], expect = -3, cap * page + 1, -2, {ora.BAD_COUNTS}
    if what == "kept":
        budget = np.array([1, 2, 1, 0, 3, 2], np.int32)
        kept = np.zeros((B, 2, 3), np.int32)
        kept[:, :, 1], kept[:, :, 2] = 1, 2
        kept[4, 1], kept[5, 0], kept[0, 0, 0] = (0, 2, 2), (1, 0, 0), 2
        expect = {ora.BAD_KEPT}
    if what == "page":
        pool.page_table[1, 0, 1], pool.page_table[4, 1, 0] = 24, -5
        n_new, expect = np.array([5, -1, 2, 40, -1, 1]), {ora.BAD_PAGE}
    if what == "page_of_growth":
        pool.page_table[0, 1, 1], expect = 99, {ora.BAD_PAGE}
    if what == "slots":
        n_slots, expect = 47, {ora.BAD_COUNTS}
    if what == "left":
        budget, kept = np.array([-1, 0, -1, 0, 1, -1], np.int32), np.zeros((B, 2, 1), np.int32)
    assert run_update(pool, n_new, n_slots, kept, budget) == expect


# ------------------------------------------------------------------ rows

@pytest.mark.parametrize("L,lists,dc,dr,page,n,layers", [(1, 0, 512, 64, 64, 1, (0, 1)), (3, 1, 128, 16, 32, 77, (1, 3)), (2, 0, 384, 48, 32, 2500, (0, 2))])
def test_rows_land_in_their_slots_and_nowhere_else(L, lists, dc, dr, page, n, layers):
    b = ngc()
    P, G = n // page + 5, L if lists else 1
    rows = normal((L, P, page, dc + dr), 1)
    pool = b.NgcLatentPool(rows.cuda(), torch.full((1, G, 1), -1, dtype=torch.int32, device="cuda"), torch.zeros((G, P), dtype=torch.uint8, device="cuda"),
                           torch.zeros((1, G), dtype=torch.int32, device="cuda"), dc, lists)
    rng = np.random.default_rng(n)
    slots = np.stack([rng.permutation(P * page)[: n + 4] for _ in range(G)]).astype(np.int32)
    slots[:, n // 2] = -1
    slots[0, -1] = P * page                                     # reported, and written nowhere
    latent, rope = normal((L, n + 4, dc), 2), normal((L, n + 4, dr), 3)
    st = b.new_status()
    b.ngc_latent_write(pool, torch.as_tensor(slots).cuda(), latent.cuda(), rope.cuda(), *layers, status=st)
    want = rows.clone().view(L, P * page, dc + dr)
    for l in range(*layers):
        s = slots[l if lists else 0]
        ok = (s >= 0) & (s < P * page)
        want[l, s[ok]] = torch.cat([latent[l, ok], rope[l, ok]], -1)
    assert torch.equal(pool.rows.cpu().view(torch.int16), want.view_as(rows).view(torch.int16))
    assert status_value(st) == (13 if (not lists or layers[0] == 0) else 0)


# ------------------------------------------------------------------ absorbed form

def run_decode(pool, H, scale, out_dtype=f32, layers=(0, None), seed=5, fill=None):
    b = ngc()
    L, B, dc, dr = pool.L, pool.B, pool.d_latent, pool.d_rope
    ql, qr = normal((L, B, H, dc), seed), normal((L, B, H, dr), seed + 1)
    out = torch.full((L, B, H, dc), 7.0 if fill is None else fill, dtype=out_dtype, device="cuda")
    ws = b.alloc_workspace(b.latent_decode_workspace_bytes(pool, H))
    ws.fill_(0xAB)
    st = b.new_status()
    b.ngc_latent_decode(pool, ql.cuda(), qr.cuda(), out, scale, *layers, ws=ws, status=st)
    torch.cuda.synchronize()
    return ql, qr, out, st


DECODE = [
    # L, lists, B, H, dc, dr, page, lens, out
    (1, 0, 1, 1, 128, 16, 32, [1], f32),
    (1, 0, 1, 16, 512, 64, 64, [700], bf16),
    (1, 0, 3, 16, 512, 64, 64, [0, 63, 65], bf16),
    (2, 1, 4, 5, 256, 32, 32, [[31, 1], [33, 64], [0, 200], [129, 128]], f32),
    (1, 0, 2, 40, 512, 64, 32, [1000, 17], f32),
    (2, 0, 2, 64, 384, 48, 64, [300, 511], bf16),
    (1, 0, 2, 128, 512, 64, 32, [257, 640], bf16),
    (1, 0, 1, 96, 128, 64, 64, [2000], f32),
    (1, 0, 70, 12, 256, 64, 64, list(range(0, 1400, 20)), bf16),
    (1, 0, 1, 16, 512, 64, 64, [9000], f32),
    (3, 2, 60, 20, 128, 32, 32, [[i, 2 * i, 100 - i] for i in range(60)], f32),
]


@pytest.mark.parametrize("i", range(len(DECODE)))
def test_decode_matches_the_definition(i):
    L, lists, B, H, dc, dr, page, lens, out_dtype = DECODE[i]
    lens = np.asarray(lens).reshape(B, -1)
    cap = max(1, -(-int(lens.max()) // page))
    n_pages = int((-(-lens // page)).sum(0).max()) + 2
    pool = random_pool(L, B, page, cap, n_pages, lens, lists, 20 + i, dc, dr)
    # rows behind the length, and pages of nobody: whatever lies there takes no part
    dead = np.ones((L, n_pages, page), bool)
    table, ln = host(pool.page_table), host(pool.lens)
    for l in range(L):
        g = l if lists else 0
        for s in range(B):
            for t in range(ln[s, g]):
                dead[l, table[s, g, t // page], t % page] = False
    rows = pool.rows.cpu()
    rows[torch.as_tensor(dead)] = torch.tensor([float("nan"), float("inf"), -float("inf"), 3e38] * ((dc + dr) // 4)).to(bf16)
    pool.rows.copy_(rows)
    scale = (128 + dr) ** -0.5
    ql, qr, out, st = run_decode(pool, H, scale, out_dtype)
    assert status_value(st) == 0
    want, bound = ora.decode(host(rows), table, ln, host(ql), host(qr), scale, lists, out_dtype is bf16)
    assert_within(out, want, bound, f"case {i}")


def test_decode_of_growing_scores_and_of_one_layer():
    """Scores that rise along the cache move the running maximum in every tile; only the range's layers are written."""
    pool = random_pool(3, 2, 64, 12, 30, [700, 130], 1, 31, 256, 64)
    ramp = torch.linspace(0.1, 6, 30 * 64).view(30, 64, 1)
    order = pool.page_table[0, 1, :11].long()
    ramp2 = torch.ones(30, 64, 1)
    ramp2[order.cpu()] = ramp[:11]
    pool.rows[1] *= ramp2.cuda().to(bf16)
    ql, qr, out, st = run_decode(pool, 28, 0.3, f32, (1, 2))
    assert status_value(st) == 0
    want, bound = ora.decode(host(pool.rows), host(pool.page_table), host(pool.lens), host(ql), host(qr), 0.3, 1)
    assert_within(out[1], want[1], bound[1])
    assert bool((out[0] == 7).all()) and bool((out[2] == 7).all())


def test_decode_reports_bad_lengths_and_pages_and_spares_the_others():
    pool = random_pool(1, 4, 32, 6, 40, [100, 150, 90, 64], 0, 33, 128, 16)
    good = [host(x) for x in (pool.rows, pool.page_table, pool.lens)]
    pool.lens[1, 0] = 6 * 32 + 1
    ql, qr, out, st = run_decode(pool, 8, 0.1)
    assert status_value(st) == 1
    want, bound = ora.decode(*good, host(ql), host(qr), 0.1, 0)
    for s in (0, 2, 3):
        assert_within(out[:, s], want[:, s], bound[:, s])
    assert bool((out[0, 1] == 7).all())
    pool.lens[1, 0] = 150
    pool.page_table[2, 0, 1] = 40
    ql, qr, out, st = run_decode(pool, 8, 0.1)
    assert status_value(st) == 11
    for s in (0, 1, 3):
        assert_within(out[:, s], want[:, s], bound[:, s])


# ------------------------------------------------------------------ expanded form

def history(T, rounds, seed, block=1):
    """(length at the round, positions kept) of a sequence: every round keeps part of what is there, in units of ``block``."""
    rng = np.random.default_rng(seed)
    alive, out, at = np.zeros(0, np.int64), [], 0
    for fired, share in rounds:
        alive = np.concatenate([alive, np.arange(at, fired)])
        at = fired
        unit = alive // block
        keep = rng.random(int(unit.max()) + 1) < share
        alive = alive[keep[unit]]
        out.append((fired, alive))
    return out


def device_history(hist, B, G, kt=None):
    """hist[b][g]: a list of (fired, kept); sequences with fewer rounds get rounds that never fire."""
    R = max(len(h) for per in hist for h in per)
    kt = kt or max(1, max(len(k) for per in hist for h in per for _, k in h))
    pos, count, total = np.full((R, B, G, kt), -1, np.int32), np.zeros((R, B, G), np.int32), np.full((R, B), 2 ** 30, np.int32)
    for s in range(B):
        for g in range(G):
            for r, (fired, kept) in enumerate(hist[s][g]):
                pos[r, s, g, : len(kept)], count[r, s, g], total[r, s] = kept, len(kept), fired
    return [torch.as_tensor(x).cuda() for x in (pos, count, total)]


class Replay:
    """Inputs of a call on whole sequences, with NaN in every row that is no token."""

    def __init__(self, L, B, H, dr, lens, spare, seed, rounds=None, lists=0, block=1, loud=4):
        b = ngc()
        self.L, self.B, self.H, self.dr, self.lens, self.lists = L, B, H, dr, list(lens), lists
        self.off = [0]
        for n in lens:
            self.off.append(self.off[-1] + n + spare)
        rows, G = self.off[-1], L if lists else 1
        self.q, self.kv, self.kr, self.go = (normal((L, rows) + s, seed + i, loud if i == 1 else 0)
                                             for i, s in enumerate([(H, 128 + dr), (H, 256), (dr,), (H, 128)]))
        for s in range(B):
            for x in (self.q, self.kv, self.kr, self.go):
                x[:, self.off[s] + self.lens[s]: self.off[s + 1]] = float("nan")
        self.hist = None if rounds is None else [[history(n, [(int(f * n), sh) for f, sh in rounds if int(f * n) > 0], seed + 100 * s + g, block) for g in range(G)]
                                                 for s, n in enumerate(self.lens)]
        self.alive = (None, None, None) if rounds is None else device_history(self.hist, B, G)
        self.seqs = b.NgcLatentSeqs(torch.tensor(self.off).cuda(), torch.tensor(self.lens, dtype=torch.int32).cuda(), max(self.lens))
        self.scale = (128 + dr) ** -0.5
        self.dev = [x.cuda() for x in (self.q, self.kv, self.kr, self.go)]

    def ws(self, backward):
        b = ngc()
        n = b.latent_replay_workspace_bytes(self.seqs, self.dev[0], self.dev[1], self.lists, 0 if self.hist is None else self.alive[0].shape[0], backward)
        w = b.alloc_workspace(n)
        if w is not None:
            w.fill_(0xAB)
        return w

    def forward(self, out_dtype=bf16, lse=True):
        b = ngc()
        self.st = b.new_status()
        self.out = torch.full((self.L, self.off[-1], self.H, 128), 7.0, dtype=out_dtype, device="cuda")
        self.lse = torch.full((self.L, self.H, self.off[-1]), 7.0, device="cuda") if lse else None
        b.ngc_latent_replay_attn(self.seqs, *self.dev[:3], self.out, self.lse, *self.alive, lists=self.lists, ws=self.ws(False), status=self.st)
        return self.out, self.lse

    def backward(self):
        b = ngc()
        self.grads = [torch.full(x.shape, 7.0, dtype=bf16, device="cuda") for x in self.dev[:3]]
        b.ngc_latent_replay_attn_backward(self.seqs, *self.dev[:3], self.out, self.lse, self.dev[3], *self.grads, *self.alive, lists=self.lists,
                                          ws=self.ws(True), status=self.st)
        return self.grads

    def strips(self):
        for l in range(self.L):
            for s in range(self.B):
                T = self.lens[s]
                if T == 0:
                    continue
                see = ora.visible(T, [] if self.hist is None else self.hist[s][l if self.lists else 0])
                yield l, s, slice(self.off[s], self.off[s] + T), see

    def check_forward(self):
        rows = np.zeros(self.off[-1], bool)
        for l, s, at, see in self.strips():
            rows[at] = True
            out, lse, ob, lb = ora.replay(host(self.q[l, at]), host(self.kv[l, at]), host(self.kr[l, at]), see, self.scale, self.out.dtype is bf16)
            assert_within(self.out[l, at], out, ob, f"out of layer {l}, sequence {s}")
            if self.lse is not None:
                assert_within(self.lse[l, :, at], lse, lb, f"lse of layer {l}, sequence {s}")
        assert bool((self.out[:, torch.as_tensor(~rows)] == 7).all()) and (self.lse is None or bool((self.lse[:, :, torch.as_tensor(~rows)] == 7).all()))

    def check_backward(self):
        rows = np.zeros(self.off[-1], bool)
        for l, s, at, see in self.strips():
            rows[at] = True
            want = ora.replay_grad(host(self.q[l, at]), host(self.kv[l, at]), host(self.kr[l, at]), see, self.scale, host(self.out[l, at]),
                                   host(self.lse[l, :, at]).astype(np.float64), host(self.go[l, at]))
            for name, g, (v, e) in zip(("q", "kv", "k_rope"), self.grads, want):
                assert_within(g[l, at], v, e, f"gradient of {name}, layer {l}, sequence {s}")
        for g in self.grads:
            assert bool((g[:, torch.as_tensor(~rows)] == 7).all())


REPLAY = [
    # L, H, dr, lens, spare, rounds (share of the sequence, share kept), lists, block
    (1, 1, 64, [1], 0, None, 0, 1),
    (1, 2, 64, [127, 128, 129], 3, None, 0, 1),
    (1, 3, 16, [0, 200, 1, 385], 1, None, 0, 1),
    (2, 2, 32, [300, 64], 0, [(0.3, 0.5), (0.6, 0.5)], 1, 1),
    (1, 2, 48, [513, 700], 5, [(0.2, 0.5), (0.5, 0.3), (0.51, 0.9), (0.8, 0.1)], 0, 32),
    (1, 1, 64, [900], 0, [(0.3, 0.0), (0.7, 0.02)], 0, 64),
    (2, 4, 64, [257], 2, [(0.5, 0.5), (0.9, 0.5)], 2, 8),
    (1, 1, 64, [1200, 40], 0, [(i / 40, 0.9) for i in range(2, 40)], 0, 1),
]


@pytest.mark.parametrize("i", range(len(REPLAY)))
@pytest.mark.parametrize("out_dtype", [bf16, f32])
def test_replay_matches_the_definition(i, out_dtype):
    L, H, dr, lens, spare, rounds, lists, block = REPLAY[i]
    r = Replay(L, len(lens), H, dr, lens, spare, 40 + i, rounds, lists, block)
    r.forward(out_dtype, lse=i % 3 != 1 or out_dtype is f32)
    r.check_forward()
    assert status_value(r.st) == 0


@pytest.mark.parametrize("i", range(len(REPLAY)))
def test_gradient_matches_the_formula(i):
    L, H, dr, lens, spare, rounds, lists, block = REPLAY[i]
    r = Replay(L, len(lens), H, dr, lens, spare, 60 + i, rounds, lists, block)
    r.forward(f32 if i % 2 else bf16)
    r.backward()
    r.check_backward()
    assert status_value(r.st) == 0


def test_gradient_matches_differences():
    """Central differences of sum(out * go) in 64 bits, along random directions of q, kv and k_rope."""
    r = Replay(1, 1, 2, 32, [150], 0, 77, [(0.4, 0.5), (0.7, 0.6)], 0, 1, loud=0)
    r.forward(f32)
    grads = [host(g).astype(np.float64)[0] for g in r.backward()]
    _, _, at, see = next(iter(r.strips()))
    x = [host(t[0]).astype(np.float64) for t in (r.q, r.kv, r.kr)]
    go = host(r.go[0]).astype(np.float64)
    rng = np.random.default_rng(5)

    def loss(*y):
        return float((ora.replay(*y, see, r.scale)[0] * go).sum())
    bounds = ora.replay_grad(*x, see, r.scale, host(r.out[0]), host(r.lse[0]).astype(np.float64), go)
    for k in range(3):
        for _ in range(3):
            d = rng.standard_normal(x[k].shape)
            h = 1e-4
            y1, y2 = list(x), list(x)
            y1[k], y2[k] = x[k] + h * d, x[k] - h * d
            numeric = (loss(*y1) - loss(*y2)) / (2 * h)
            # roundings of the kernel's values count each with its sign; the differences are good to h^2
            assert abs(numeric - float((grads[k] * d).sum())) <= float((bounds[k][1] * np.abs(d)).sum()) + 1e-5 * abs(numeric) + 1e-4


def test_scores_that_rise_and_fall_along_the_sequence():
    """Keys that grow along the sequence move the running maximum in every tile; then ones that shrink."""
    for sign in (1, -1):
        r = Replay(1, 1, 2, 64, [700], 0, 80, None)
        ramp = torch.linspace(0.05, 3, 700)[:: sign] if sign > 0 else torch.linspace(0.05, 3, 700).flip(0)
        r.kv[0, :, :, :128] = (r.kv[0, :, :, :128].float() * ramp[:, None, None]).to(bf16)
        r.dev[1].copy_(r.kv)
        r.forward(f32)
        r.check_forward()
        r.backward()
        r.check_backward()


def test_replay_reports_bad_lists_and_lengths_and_spares_other_sequences():
    r = Replay(1, 3, 1, 64, [200, 300, 150], 0, 90, [(0.5, 0.5)])
    r.alive[0][0, 1, 0, 3] = 299                                # not there yet at the round
    r.forward()
    assert status_value(r.st) == 3
    r.hist[1][0] = [(f, [x for i, x in enumerate(k) if i != 3]) for f, k in r.hist[1][0]]
    r.check_forward()
    r = Replay(1, 3, 1, 64, [200, 300, 150], 0, 90, [(0.5, 0.5)])
    r.seqs.lens[1] = 301
    r.forward()
    r.backward()
    assert status_value(r.st) == 1
    assert bool((r.out[:, 200:500] == 7).all()) and all(bool((g[:, 200:500] == 7).all()) for g in r.grads)


# ------------------------------------------------------------------ together

def test_prompts_rounds_and_steps_of_a_rollout_agree_with_the_replay():
    """Prompts admitted to the pool, decode steps, an eviction round in between: with the projections applied, every step's absorbed
    attention is the expanded replay's row of that token."""
    from paper_2604_18002_b200.rollout import NgcLatentRollout
    b = ngc()
    L, B, H, dc, dr, page = 2, 3, 4, 256, 32, 32
    prompt, steps, scale = [70, 33, 100], 75, (128 + dr) ** -0.5
    T = [p + steps for p in prompt]
    latent, rope = [normal((L, n, dc), 300 + i) for i, n in enumerate(T)], [normal((L, n, dr), 320 + i) for i, n in enumerate(T)]
    g = torch.Generator().manual_seed(7)
    U, W = ((torch.randn((L, H, 128, dc), generator=g) / dc ** 0.5).to(bf16) for _ in range(2))
    qn, qr = [normal((L, n, H, 128), 340 + i) for i, n in enumerate(T)], [normal((L, n, H, dr), 360 + i) for i, n in enumerate(T)]
    ro = NgcLatentRollout(L, B, H, dc, dr, n_pages=24, pages_cap=8, max_new=sum(prompt), scale=scale, page=page, lists=b.LISTS_PER_LAYER)
    ro.update(torch.tensor(prompt, dtype=torch.int32).cuda())
    ro.write(torch.cat([x[:, :p] for x, p in zip(latent, prompt)], 1).cuda(), torch.cat([x[:, :p] for x, p in zip(rope, prompt)], 1).cuda())
    got = [torch.zeros((L, n, H, 128)) for n in T]
    n_new = torch.ones(B, dtype=torch.int32).cuda()
    hist = [[[] for _ in range(L)] for _ in range(B)]
    rounds_at = {20: 2, 45: 3}
    pos = [[list(range(p)) for _ in range(L)] for p in prompt]              # original positions of the alive rows, page by page
    for i in range(steps):
        now = [p + i for p in prompt]
        if i in rounds_at:
            keep = rounds_at[i]
            logits = torch.randn((B, L, 8), generator=g).cuda()
            n = torch.tensor([[-(-len(pos[s][l]) // page) for l in range(L)] for s in range(B)])
            for s in range(B):
                for l in range(L):
                    logits[s, l, int(n[s, l]):] = -float("inf")             # a layer may be a page short of the others
            ro.evict(logits, n.max(1).values.to(torch.int32).cuda(), None, torch.full((B,), keep, dtype=torch.int32).cuda(), 11, i, n_new)
            kept = ro.kept_sorted.cpu()
            for s in range(B):
                for l in range(L):
                    units = kept[s, l, :keep].tolist()
                    pos[s][l] = [x for u in units for x in pos[s][l][u * page: (u + 1) * page]]
                    hist[s][l].append((now[s], np.array(pos[s][l])))
        else:
            ro.update(n_new)
        for s in range(B):
            for l in range(L):
                pos[s][l].append(now[s])
        new_l, new_r = torch.zeros((L, sum(prompt), dc), dtype=bf16), torch.zeros((L, sum(prompt), dr), dtype=bf16)
        for s in range(B):
            new_l[:, s], new_r[:, s] = latent[s][:, now[s]], rope[s][:, now[s]]
        out = torch.zeros((L, B, H, dc), device="cuda")
        q = torch.stack([torch.einsum("lhd,lhdc->lhc", qn[s][:, now[s]].float(), U.float()) for s in range(B)], 1).to(bf16).cuda()
        r = torch.stack([qr[s][:, now[s]] for s in range(B)], 1).cuda()
        for l in range(L):                                                  # as a model calls them
            ro.write(new_l.cuda(), new_r.cuda(), l, l + 1)
            ro.decode(q, r, out, l, l + 1)
        for s in range(B):
            got[s][:, now[s]] = torch.einsum("lhc,lhdc->lhd", out[:, s].cpu(), W.float())
    ro.check_status()
    assert [[len(x) for x in per] for per in pos] == host(ro.pool.lens).tolist()
    # the training pass over the same tokens
    rows = sum(T)
    kv = torch.cat([torch.cat([torch.einsum("ltc,lhdc->lthd", x.float(), w.float()).to(bf16) for w in (U, W)], -1) for x in latent], 1)
    off = [0] + np.cumsum(T).tolist()
    seqs = b.NgcLatentSeqs(torch.tensor(off).cuda(), torch.tensor(T, dtype=torch.int32).cuda(), max(T))
    alive = device_history(hist, B, L)
    q = torch.cat([torch.cat([a, c], -1) for a, c in zip(qn, qr)], 1).cuda()
    out = torch.zeros((L, rows, H, 128), device="cuda")
    st = b.new_status()
    ws = b.alloc_workspace(b.latent_replay_workspace_bytes(seqs, q, kv.cuda(), b.LISTS_PER_LAYER, alive[0].shape[0]))
    b.ngc_latent_replay_attn(seqs, q, kv.cuda(), torch.cat(rope, 1).cuda(), out, None, *alive, lists=b.LISTS_PER_LAYER, ws=ws, status=st)
    assert status_value(st) == 0
    for s in range(B):
        a, c = got[s][:, prompt[s]:], out[:, off[s] + prompt[s]: off[s + 1]].cpu()
        # roundings on the way: the absorbed query, keys, values and probabilities, each half a step of bf16 (2**-8); scores are sums of
        # some 300 products of size 1 / 13 with independent roundings, so they move by 0.01 or so, outputs by a few hundredths of their size
        assert float((a - c).norm() / c.norm()) <= 0.02
