"""Cases that measure the operators of latent attention: the pages of a common pool and their slot maps,
the rows of new tokens, attention of one new token over the pool (absorbed form), and attention of whole
sequences under their history of evictions with its gradient (expanded form).

``run`` computes a case in plain torch operations (``own`` false) or through the library's entry points
(``own`` true); both take what ``prepare`` gives.  ``exact`` is the attention, forward and backward, from
its definition in 64 bits; the other operators move rows or compute whole numbers.
"""
from __future__ import annotations

import math
import types

import torch

own = False


def listed():
    return [
        # one decode step of a batch: a page for every 64th token, the slot of each
        dict(name="pool_step", op="pool", layers=1, lists=0, batch=64, page=64, t_lo=1024, t_hi=4096, new_lo=1, new_hi=1, keep=0.0,
             evicting=0.0, finished=0.0),
        # an eviction round on every layer's own pages, with finished rollouts leaving and the next token in the same call
        dict(name="pool_round", op="pool", layers=28, lists=1, batch=64, page=32, t_lo=1500, t_hi=3000, new_lo=1, new_hi=1, keep=0.5,
             evicting=0.8, finished=0.05),
        # prompts of many lengths admitted into an empty pool
        dict(name="pool_admit", op="pool", layers=28, lists=1, batch=256, page=64, t_lo=0, t_hi=0, new_lo=200, new_hi=2000, keep=0.0,
             evicting=0.0, finished=0.0),
        # the new rows of one decode step, layer by layer
        dict(name="write_step", op="write", layers=1, lists=0, tokens=64, padding=0, dc=512, dr=64, page=64, n_pages=2048),
        # the rows of admitted prompts, several layers in a call, odd count, some slots unused
        dict(name="write_prompts", op="write", layers=8, lists=1, tokens=32113, padding=655, dc=512, dr=64, page=32, n_pages=1400),
        # one rollout, one layer: latency
        dict(name="decode_one", op="decode", layers=1, lists=0, batch=1, heads=16, dc=512, dr=64, page=64, t_lo=700, t_hi=700),
        # a serving step of a model that calls its layers one by one: ragged rollouts, 16 heads
        dict(name="decode_b64", op="decode", layers=1, lists=0, batch=64, heads=16, dc=512, dr=64, page=64, t_lo=1024, t_hi=4096),
        # all heads of a large model on one device, two layers with pages of their own, long caches
        dict(name="decode_128_heads", op="decode", layers=2, lists=1, batch=24, heads=128, dc=512, dr=64, page=32, t_lo=2048, t_hi=8192),
        # prompts: causal, ragged, odd lengths
        dict(name="replay_prompts", op="replay", layers=1, lists=0, batch=4, heads=16, dr=64, t_lo=333, t_hi=1111, block=32, budget=0, step=0, rounds=0),
        # the training pass over long rollouts: a round every 1024 tokens keeps 1024
        dict(name="replay_rollouts", op="replay", layers=1, lists=0, batch=2, heads=16, dr=64, t_lo=6500, t_hi=8192, block=64, budget=1024, step=1024, rounds=7),
        # gradients of a batch of prompts
        dict(name="grad_prompts", op="grad", layers=1, lists=0, batch=4, heads=16, dr=64, t_lo=333, t_hi=1111, block=32, budget=0, step=0, rounds=0),
        # gradients of the training pass over long rollouts
        dict(name="grad_rollouts", op="grad", layers=1, lists=0, batch=2, heads=16, dr=64, t_lo=6500, t_hi=8192, block=64, budget=1024, step=1024, rounds=7),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["pool", "write", "decode", "decode", "replay", "grad"])
    lists = rng.choice([0, 1])
    layers = rng.choice([1, 1, 2, 3])
    if op == "pool":
        t_hi = rng.choice([0, _log(rng, 1, 8192)])
        new_hi = rng.choice([1, 1, _log(rng, 1, 2048)])
        evict = rng.random() < 0.5
        layers, batch = rng.choice([1, 2, 7, 28]), _log(rng, 1, 256)
        while batch * layers * (t_hi + new_hi) > 28 * 256 * 1100:
            batch //= 2
        return dict(op=op, layers=layers, lists=lists, batch=batch, page=rng.choice([32, 64]),
                    t_lo=rng.choice([0, t_hi // 2, t_hi]), t_hi=t_hi, new_lo=rng.choice([0, 1, new_hi]), new_hi=new_hi,
                    keep=rng.choice([0.0, 0.25, 0.5, 0.9]) if evict else 0.0, evicting=rng.choice([0.5, 1.0]) if evict else 0.0,
                    finished=rng.choice([0.0, 0.2]))
    if op == "write":
        return dict(op=op, layers=layers, lists=lists, tokens=_log(rng, 1, 32768), padding=rng.choice([0, rng.randrange(300)]),
                    dc=rng.choice([128, 256, 384, 512]), dr=rng.choice([16, 32, 48, 64]), page=rng.choice([32, 64]), n_pages=_log(rng, 1100, 3000))
    if op == "decode":
        c = dict(op=op, layers=layers, lists=lists, batch=_log(rng, 1, 128), heads=rng.choice([1, 5, 8, 12, 16, 20, 28, 32, 40, 64, 96, 128]),
                 dc=rng.choice([128, 256, 384, 512, 512, 512]), dr=rng.choice([16, 32, 48, 64, 64, 64]), page=rng.choice([32, 64]),
                 t_hi=_log(rng, 1, 65536))
        c["t_lo"] = rng.choice([0, c["t_hi"] // 2, c["t_hi"]])
        while c["batch"] * c["layers"] * c["t_hi"] * max(c["heads"], 16) > 2 * 24 * 5120 * 128:
            if c["batch"] > 1:
                c["batch"] //= 2
            else:
                c["t_hi"] //= 2
                c["t_lo"] = min(c["t_lo"], c["t_hi"])
        return c
    # (the gradients of a handful of tokens are differences of nearly equal numbers: nothing to compare)
    t_hi = _log(rng, 1 if op == "replay" else 48, 8192)
    c = dict(op=op, layers=rng.choice([1, 1, 2]), lists=lists, batch=_log(rng, 1, 16), heads=rng.choice([1, 3, 8, 12, 16, 28, 32]),
             dr=rng.choice([16, 32, 48, 64, 64, 64]), t_lo=rng.choice([max(1, t_hi // 3), t_hi]), t_hi=t_hi, block=rng.choice([1, 8, 32, 64]))
    budget, step = 64 * _log(rng, 1, 32), 64 * _log(rng, 1, 32)
    rounds = rng.choice([0, 1]) * min(15, max(0, (t_hi - budget) // step))
    c.update(budget=budget if rounds else 0, step=step if rounds else 0, rounds=rounds)
    while c["batch"] * c["layers"] * c["heads"] * t_hi * t_hi > 16 * 2 * 7000 * 7000 and c["batch"] > 1:
        c["batch"] //= 2
    while c["batch"] * c["layers"] * c["heads"] * t_hi * t_hi > 16 * 2 * 7000 * 7000 and c["heads"] > 1:
        c["heads"] //= 2
    c["heads"] = max(1, c["heads"])
    return c


# ---------------------------------------------------------------- inputs, from the seed alone

def _spread(lo, hi, n):
    """n whole numbers from lo to hi, evenly spaced: the same sum whatever their order."""
    return [hi if n == 1 else lo + (hi - lo) * i // (n - 1) for i in range(n)]


def _lists(c):
    return c["layers"] if c["lists"] else 1


def _new(c):
    done = int(c["finished"] * c["batch"])
    return [-1] * done + _spread(c["new_lo"], c["new_hi"], c["batch"])[done:]


def _pages(tokens, page):
    return -(-tokens // page)


def _shuffle(values, g):
    t = torch.tensor(values, dtype=torch.int64)
    return t[torch.randperm(len(values), generator=g)]


def _pool_inputs(c, s, g):
    B, G, page = c["batch"], _lists(c), c["page"]
    lens = _shuffle(_spread(c["t_lo"], c["t_hi"], B), g)
    new = _shuffle(_new(c), g)                                                # -1: finished, everything goes back to the pool
    have = _pages(lens, page)
    # what the earlier rounds left: on some layers a short last page, on others a full one
    lens_g = lens[:, None].repeat(1, G)
    if G > 1 and c["t_hi"]:
        lens_g = torch.where(torch.rand((B, G), generator=g) < 0.5, lens_g, have[:, None] * page)
    cap = _pages(c["t_hi"] + page + c["new_hi"], page) + 1
    n_pages = int((_pages(lens, page) + 1 + _pages(new.clamp(min=0), page)).sum()) + 7
    table = torch.full((B, G, cap), -1, dtype=torch.int32)
    used = torch.zeros((G, n_pages), dtype=torch.uint8)
    first = torch.cumsum(have, 0) - have
    j = torch.arange(cap)
    mine = j < have[:, None]
    for gi in range(G):
        order = torch.randperm(n_pages, generator=g)                          # pages of a pool in use lie anywhere
        row = order[(first[:, None] + j).clamp(max=n_pages - 1)]
        table[:, gi] = torch.where(mine, row, -1).to(torch.int32)
        used[gi, order[: int(have.sum())]] = 1
    parts = [table.flatten().view(torch.uint8), lens_g.to(torch.int32).flatten().view(torch.uint8), used.flatten()]
    s.start = torch.cat(parts).cuda()                                         # the pool's books before the call, in one piece
    s.live = s.start.clone()
    a, b = parts[0].numel(), parts[0].numel() + parts[1].numel()
    s.table = s.live[:a].view(torch.int32).view(B, G, cap)
    s.lens = s.live[a:b].view(torch.int32).view(B, G)
    s.used = s.live[b:].view(G, n_pages)
    s.n_new = new.to(torch.int32).cuda()
    s.slots = torch.empty((G, max(1, sum(max(n, 0) for n in _new(c)))), dtype=torch.int32, device="cuda")
    s.first = torch.empty((B + 1,), dtype=torch.int32, device="cuda")
    s.kept = s.budget = None
    if c["evicting"]:
        budget = (have.double() * c["keep"]).ceil().long()
        k_max = max(1, int(budget.max()))
        rank = torch.where(j < have[:, None, None], torch.rand((B, G, cap), generator=g), 2.0).argsort(-1)[..., :k_max]
        kept = torch.where(torch.arange(k_max) < budget[:, None, None], rank, cap).sort(-1).values
        s.kept = torch.where(kept < cap, kept, -1).to(torch.int32).cuda()
        idle = torch.rand((B,), generator=g) >= c["evicting"]
        s.budget = torch.where(idle, -1, budget).to(torch.int32).cuda()       # -1: no round for this sequence
    if own:
        s.rows = torch.empty((c["layers"], n_pages, page, 144), dtype=torch.bfloat16, device="cuda")


def _history(c, g, R, B, G):
    """Kept lists of R rounds in original positions, as the replay calls take them: ``budget`` tokens in whole units stay."""
    block, n_keep, n_step = c["block"], c["budget"] // c["block"], c["step"] // c["block"]
    alive = torch.empty((B, G, 0), dtype=torch.int64)
    total, lists = 0, []
    for r in range(R):
        new_total = c["budget"] + c["step"] * (r + 1)
        alive = torch.cat([alive, torch.arange(total // block, new_total // block).expand(B, G, -1)], -1)
        keep = torch.rand(alive.shape, generator=g).argsort(-1)[..., :n_keep].sort(-1).values
        alive = torch.gather(alive, -1, keep)
        lists.append((alive[..., None] * block + torch.arange(block)).flatten(-2))
        total = new_total
    tb = torch.tensor([c["budget"] + c["step"] * (r + 1) for r in range(R)], dtype=torch.int32)
    return torch.stack(lists).to(torch.int32).cuda(), torch.full((R, B, G), n_keep * block, dtype=torch.int32).cuda(), tb[:, None].repeat(1, B).cuda()


def _inputs(c, seed):
    g = torch.Generator().manual_seed(int(seed) * 7919 + 1)
    gd = torch.Generator(device="cuda").manual_seed(int(seed) * 104729 + 3)
    s = types.SimpleNamespace(case=c)
    op, L, G = c["op"], c["layers"], _lists(c)

    def normal(*shape):
        return torch.empty(shape, dtype=torch.bfloat16, device="cuda").normal_(generator=gd)

    if op == "pool":
        _pool_inputs(c, s, g)
        return s
    if op == "write":
        n, total, P, page = c["tokens"], c["tokens"] + c["padding"], c["n_pages"], c["page"]
        s.rows = normal(L, P, page, c["dc"] + c["dr"])
        slots = torch.stack([torch.randperm(P, generator=g) for _ in range(G)])[:, : _pages(n, page)]
        slots = (slots[..., None] * page + torch.arange(page)).flatten(-2)[:, :n]
        s.slots = torch.full((G, total), -1, dtype=torch.int32)
        s.slots[:, :n] = slots
        s.slots = s.slots.cuda()
        s.latent, s.rope = normal(L, total, c["dc"]), normal(L, total, c["dr"])
        if own:
            s.table, s.lens = torch.full((1, G, 1), -1, dtype=torch.int32, device="cuda"), torch.zeros((1, G), dtype=torch.int32, device="cuda")
            s.used = torch.ones((G, P), dtype=torch.uint8, device="cuda")
        return s
    if op == "decode":
        B, H, page, dc, dr = c["batch"], c["heads"], c["page"], c["dc"], c["dr"]
        lens = _shuffle(_spread(c["t_lo"], c["t_hi"], B), g)
        have = _pages(lens, page)
        cap, P = max(1, int(have.max())), max(1, int(have.sum()))
        first = torch.cumsum(have, 0) - have
        table = torch.full((B, G, cap), -1, dtype=torch.int32)
        j = torch.arange(cap)
        for gi in range(G):
            row = torch.randperm(P, generator=g)[(first[:, None] + j).clamp(max=P - 1)]
            table[:, gi] = torch.where(j < have[:, None], row, -1).to(torch.int32)
        s.table, s.lens = table.cuda(), lens[:, None].repeat(1, G).to(torch.int32).cuda()
        s.rows = normal(L, P, page, dc + dr)
        s.rows[..., :4] *= 4                                                  # a few loud channels, as trained models have
        s.ql, s.qr = normal(L, B, H, dc), normal(L, B, H, dr)
        s.scale = 1.0 / math.sqrt(128 + dr)
        s.out = torch.zeros((L, B, H, dc), dtype=torch.bfloat16, device="cuda")
        if own:
            s.used = torch.ones((G, P), dtype=torch.uint8, device="cuda")
        return s
    B, H, dr, R = c["batch"], c["heads"], c["dr"], c["rounds"]
    lens = _shuffle(_spread(c["t_lo"], c["t_hi"], B), g)
    cap = lens + torch.arange(B) % 4                                          # a few spare rows between the sequences
    s.host_lens = lens.tolist()
    s.host_off = [0] + torch.cumsum(cap, 0).tolist()
    s.seq_off, s.lens = torch.tensor(s.host_off).cuda(), lens.to(torch.int32).cuda()
    rows = s.host_off[-1]
    s.q, s.kv, s.kr = normal(L, rows, H, 128 + dr), normal(L, rows, H, 256), normal(L, rows, dr)
    s.kv[..., :4] *= 4
    s.scale = 1.0 / math.sqrt(128 + dr)
    s.alive = _history(c, g, R, B, G) if R else (None, None, None)
    s.out = torch.zeros((L, rows, H, 128), dtype=torch.bfloat16, device="cuda")
    s.lse = torch.zeros((L, H, rows), dtype=torch.float32, device="cuda")
    if op == "grad":
        s.go = normal(L, rows, H, 128)
        s.gq, s.gkv, s.gkr = torch.zeros_like(s.q), torch.zeros_like(s.kv), torch.zeros_like(s.kr)
        _plain_replay(s)                                                      # a training step has the forward's outputs in hand
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:
        from paper_2604_18002_b200 import binding as ngc
        s.status = ngc.new_status()
        if case["op"] in ("pool", "write", "decode"):
            s.pool = ngc.NgcLatentPool(s.rows, s.table, s.used, s.lens, case.get("dc", 128), case["lists"])
        if case["op"] == "decode":
            s.ws = ngc.alloc_workspace(ngc.latent_decode_workspace_bytes(s.pool, case["heads"]))
        if case["op"] in ("replay", "grad"):
            s.seqs = ngc.NgcLatentSeqs(s.seq_off, s.lens, max(s.host_lens))
            s.ws = ngc.alloc_workspace(ngc.latent_replay_workspace_bytes(s.seqs, s.q, s.kv, _lists(case), backward=case["op"] == "grad"))
    return s


# ---------------------------------------------------------------- one pass

def run(state):
    return (_OWN if own else _PLAIN)[state.case["op"]](state)


def _own_pool(s):
    from paper_2604_18002_b200 import binding as ngc
    s.live.copy_(s.start)                                                     # back to the books before the call
    ngc.ngc_pool_update(s.pool, s.n_new, s.slots, s.first, kept_sorted=s.kept, budget=s.budget, status=s.status)
    return [s.table, s.used, s.lens, s.slots, s.first]


def _own_write(s):
    from paper_2604_18002_b200 import binding as ngc
    ngc.ngc_latent_write(s.pool, s.slots, s.latent, s.rope, status=s.status)
    return s.rows


def _own_decode(s):
    from paper_2604_18002_b200 import binding as ngc
    ngc.ngc_latent_decode(s.pool, s.ql, s.qr, s.out, s.scale, ws=s.ws, status=s.status)
    return s.out


def _own_replay(s):
    from paper_2604_18002_b200 import binding as ngc
    ngc.ngc_latent_replay_attn(s.seqs, s.q, s.kv, s.kr, s.out, s.lse, *s.alive, lists=s.case["lists"], scale=s.scale, ws=s.ws, status=s.status)
    return [s.out, s.lse]


def _own_grad(s):
    from paper_2604_18002_b200 import binding as ngc
    ngc.ngc_latent_replay_attn_backward(s.seqs, s.q, s.kv, s.kr, s.out, s.lse, s.go, s.gq, s.gkv, s.gkr, *s.alive, lists=s.case["lists"],
                                        scale=s.scale, ws=s.ws, status=s.status)
    return [s.gq, s.gkv, s.gkr]


_OWN = dict(pool=_own_pool, write=_own_write, decode=_own_decode, replay=_own_replay, grad=_own_grad)


def _plain_pool(s):
    page = s.case["page"]
    s.live.copy_(s.start)
    B, G, cap = s.table.shape
    table, lens = s.table.long(), s.lens.long()
    have = (lens + page - 1) // page
    j = torch.arange(cap, device="cuda")
    P = s.used.shape[1]
    used = torch.cat([s.used.bool(), s.used.new_zeros((G, 1)).bool()], -1)    # a place behind the pool for entries that name no page
    gi = torch.arange(G, device="cuda")[None, :, None].expand(B, G, cap)

    def mark(row, value):
        used[gi, torch.where(row >= 0, row, P)] = value

    if s.kept is not None:
        kept, n = s.kept.long(), s.budget.long()[:, None]
        short = have * page - lens                                            # what the last page lacks
        last = torch.where(n > 0, torch.gather(kept, -1, (n[:, :, None] - 1).clamp(min=0).expand(B, G, 1))[..., 0], -1)
        kept_len = n * page - torch.where(last == have - 1, short, 0)
        full = torch.full_like(table, -1)
        full[..., : kept.shape[-1]] = torch.where(kept >= 0, torch.gather(table, -1, kept.clamp(min=0)), -1)
        mark(torch.where(n[:, :, None] >= 0, table, -1), False)
        table = torch.where(n[:, :, None] >= 0, full, table)
        lens = torch.where(n >= 0, kept_len, lens)
        mark(table, True)
    done = (s.n_new < 0)[:, None]
    mark(torch.where(done[:, :, None], table, -1), False)
    table = torch.where(done[:, :, None], -1, table)
    lens = torch.where(done, 0, lens)
    new = s.n_new.long().clamp(min=0)
    have = (lens + page - 1) // page
    need = (lens + new[:, None] + page - 1) // page - have
    rank = (torch.cumsum(need, 0) - need)[:, :, None] + j - have[:, :, None]  # of the free pages, for entry j
    free = torch.sort(used[:, :P].to(torch.uint8), dim=-1, stable=True).indices      # [G][pages], the free ones first
    fresh = (j >= have[:, :, None]) & (j < (have + need)[:, :, None])
    table = torch.where(fresh, torch.gather(free.expand(B, G, -1), -1, rank.clamp(0, free.shape[-1] - 1)), table)
    mark(torch.where(fresh, table, -1), True)
    first = torch.cumsum(new, 0)
    s.first[0] = 0
    s.first[1:] = first
    i = torch.arange(s.slots.shape[1], device="cuda")
    b = torch.searchsorted(first, i, right=True).clamp(max=B - 1)
    pos = lens[b] + (i - (first - new)[b])[:, None]                           # [slots][G]
    slot = torch.gather(table[b], -1, (pos // page).clamp(max=cap - 1)[..., None])[..., 0] * page + pos % page
    s.slots.copy_(torch.where((i < first[-1])[:, None], slot, -1).t())
    s.table.copy_(table)
    s.used.copy_(used[:, :P])
    s.lens.copy_(lens + new[:, None])
    return [s.table, s.used, s.lens, s.slots, s.first]


def _plain_write(s):
    c = s.case
    for l in range(c["layers"]):
        slots = s.slots[l if c["lists"] else 0, : c["tokens"]].long()         # the others are unused
        flat = s.rows[l].view(-1, c["dc"] + c["dr"])
        flat[slots, : c["dc"]] = s.latent[l, : c["tokens"]]
        flat[slots, c["dc"]:] = s.rope[l, : c["tokens"]]
    return s.rows


def _plain_decode(s):
    c = s.case
    L, B, H, dc, page = c["layers"], c["batch"], c["heads"], c["dc"], c["page"]
    cap = s.table.shape[-1]
    live = torch.arange(cap * page, device="cuda") < s.lens.long()[..., None]  # [B][G][T]
    part = max(1, 2 ** 29 // (cap * page * (dc + H)))                         # sequences at a time
    for l in range(L):
        gi = l if c["lists"] else 0
        for b0 in range(0, B, part):
            at = slice(b0, b0 + part)
            x = s.rows[l][s.table[at, gi].long().clamp(min=0)].flatten(1, 2).float()
            x = torch.where(live[at, gi, :, None], x, 0.0)
            q = torch.cat([s.ql[l, at], s.qr[l, at]], -1).float()
            z = torch.where(live[at, gi, None], (q @ x.transpose(-1, -2)) * s.scale, -math.inf)
            z = torch.exp(z - z.amax(-1, keepdim=True).clamp(min=-1e30))
            s.out[l, at] = ((z @ x[..., :dc]) / z.sum(-1, keepdim=True).clamp(min=1e-30)).to(s.out.dtype)
    return s.out


def _gone(s, l, b):
    """Sequence length at the round that evicted each token of sequence b, on the list of layer l."""
    T = s.host_lens[b]
    pos, _, total = s.alive
    gone = torch.full((T,), 2 ** 31 - 1, device="cuda")
    if pos is None:
        return gone
    t = torch.arange(T, device="cuda")
    for r in range(pos.shape[0] - 1, -1, -1):
        there = torch.zeros((max(T, int(s.case["t_hi"])) + 1,), dtype=torch.bool, device="cuda")
        there[pos[r, b, l if s.case["lists"] else 0].long()] = True
        gone = torch.where((t < total[r, b]) & ~there[:T], total[r, b].long(), gone)
    return gone


def _strips(s):
    """Every (layer, sequence): its rows, and which keys each query sees."""
    for l in range(s.case["layers"]):
        for b, T in enumerate(s.host_lens):
            t = torch.arange(T, device="cuda")
            see = (t[None, :] <= t[:, None]) & (t[:, None] < _gone(s, l, b)[None, :])
            yield l, slice(s.host_off[b], s.host_off[b] + T), see


def _plain_replay(s):
    for l, at, see in _strips(s):
        for h in range(s.case["heads"]):
            q, k, v = s.q[l, at, h].float(), torch.cat([s.kv[l, at, h, :128], s.kr[l, at]], -1).float(), s.kv[l, at, h, 128:].float()
            z = torch.where(see, (q @ k.t()) * s.scale, -math.inf)
            m = z.amax(-1, keepdim=True)
            p = torch.exp(z - m)
            total = p.sum(-1, keepdim=True)
            s.out[l, at, h] = ((p @ v) / total).to(s.out.dtype)
            s.lse[l, h, at] = (m + torch.log(total))[:, 0]
    return [s.out, s.lse]


def _plain_grad(s):
    for l, at, see in _strips(s):
        dr = torch.zeros((see.shape[0], s.case["dr"]), device="cuda")
        for h in range(s.case["heads"]):
            q, k, v = s.q[l, at, h].float(), torch.cat([s.kv[l, at, h, :128], s.kr[l, at]], -1).float(), s.kv[l, at, h, 128:].float()
            go = s.go[l, at, h].float()
            p = torch.where(see, torch.exp((q @ k.t()) * s.scale - s.lse[l, h, at, None]), 0.0)
            delta = (go * s.out[l, at, h].float()).sum(-1, keepdim=True)
            dz = p * (go @ v.t() - delta) * s.scale
            s.gq[l, at, h] = (dz @ k).to(s.gq.dtype)
            dk = dz.t() @ q
            s.gkv[l, at, h] = torch.cat([dk[:, :128], p.t() @ go], -1).to(s.gkv.dtype)
            dr += dk[:, 128:]
        s.gkr[l, at] = dr.to(s.gkr.dtype)
    return [s.gq, s.gkv, s.gkr]


_PLAIN = dict(pool=_plain_pool, write=_plain_write, decode=_plain_decode, replay=_plain_replay, grad=_plain_grad)


# ---------------------------------------------------------------- what a pass cannot do without

def work(case):
    c = case
    op, L, G = c["op"], c["layers"], _lists(c)
    if op == "pool":
        # the books of every list: lengths and new table entries written, one byte a page of the pool, kept pages, and the slots
        have, new = [_pages(t, c["page"]) for t in _spread(c["t_lo"], c["t_hi"], c["batch"])], [max(n, 0) for n in _new(c)]
        tokens, pages = sum(new), sum(have)
        return {"bytes": G * (4 * tokens + 4 * (pages if c["evicting"] else 0) + 4 * _pages(tokens, c["page"]) + 12 * c["batch"] + pages + _pages(tokens, c["page"])), "flops": 0}
    if op == "write":
        return {"bytes": L * c["tokens"] * (c["dc"] + c["dr"]) * 4 + 4 * G * c["tokens"], "flops": 0}
    if op == "decode":
        rows = L * sum(_spread(c["t_lo"], c["t_hi"], c["batch"]))
        width, heads = c["dc"] + c["dr"], L * c["batch"] * c["heads"]
        return {"bytes": rows * width * 2 + heads * (width * 2 + c["dc"] * 2), "flops": 2 * (width + c["dc"]) * rows * c["heads"]}
    tokens, pairs = 0, 0
    for T in _spread(c["t_lo"], c["t_hi"], c["batch"]):
        ends = [0] + [c["budget"] + c["step"] * (r + 1) for r in range(c["rounds"])] + [T]
        for i in range(len(ends) - 1):
            a, e = min(ends[i], T), min(ends[i + 1], T)
            kept = (c["budget"] // c["block"]) * c["block"] if i else 0
            pairs += (e - a) * kept + (e - a) * (e - a + 1) // 2
        tokens += T
    H, dq = c["heads"], 128 + c["dr"]
    io = L * tokens * (H * dq + H * 256 + c["dr"]) * 2                        # queries, keys and values, rope rows
    if op == "replay":
        return {"bytes": io + L * tokens * H * (2 * 128 + 4), "flops": 2 * (dq + 128) * pairs * L * H}
    return {"bytes": 2 * io + L * tokens * H * (2 * 256 + 4), "flops": 2 * (3 * dq + 2 * 128) * pairs * L * H}


# ---------------------------------------------------------------- the attention from its definition, in 64 bits

def _seen(s, l, b):
    """[T][T] truth table: a simulation of the cache, segment of queries by segment."""
    T = s.host_lens[b]
    pos, count, total = s.alive
    see = torch.ones((T, T), dtype=torch.bool, device="cuda").tril()
    for r in range(0 if pos is None else pos.shape[0]):
        fired = int(total[r, b])
        if fired >= T:
            break
        gi = l if s.case["lists"] else 0
        cache = torch.zeros((fired,), dtype=torch.bool, device="cuda")
        cache[pos[r, b, gi, : int(count[r, b, gi])].long()] = True
        until = min(T, int(total[r + 1, b])) if r + 1 < pos.shape[0] else T
        see[fired:until, :fired] = cache
    return see


def exact(case, seed):
    c = case
    if c["op"] in ("pool", "write"):
        return None
    s = _inputs(c, seed)
    if c["op"] == "decode":
        out = torch.zeros(s.out.shape, dtype=torch.float64, device="cuda")
        if c["layers"] * c["batch"] > 4096:
            return None
        lens = s.lens.tolist()
        for l in range(c["layers"]):
            for b in range(c["batch"]):
                gi = l if c["lists"] else 0
                T = lens[b][gi]
                if T == 0:
                    continue
                x = s.rows[l, s.table[b, gi, : _pages(T, c["page"])].long()].reshape(-1, c["dc"] + c["dr"])[:T].double()
                z = (s.ql[l, b].double() @ x[:, : c["dc"]].t() + s.qr[l, b].double() @ x[:, c["dc"]:].t()) * s.scale
                out[l, b] = torch.softmax(z, -1) @ x[:, : c["dc"]]
        return out
    grad = c["op"] == "grad"
    out = torch.zeros(s.out.shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros(s.lse.shape, dtype=torch.float64, device="cuda")
    gq, gkv, gkr = (torch.zeros(t.shape, dtype=torch.float64, device="cuda") for t in (s.q, s.kv, s.kr)) if grad else (None, None, None)
    for l in range(c["layers"]):
        for b, T in enumerate(s.host_lens):
            see, o = _seen(s, l, b), s.host_off[b]
            for h in range(c["heads"]):
                q, kv, kr = s.q[l, o:o + T, h].double(), s.kv[l, o:o + T, h].double(), s.kr[l, o:o + T].double()
                z = (q[:, :128] @ kv[:, :128].t() + q[:, 128:] @ kr.t()) * s.scale
                z.masked_fill_(~see, -math.inf)
                lse[l, h, o:o + T] = torch.logsumexp(z, -1)
                p = torch.exp(z - lse[l, h, o:o + T, None])
                out[l, o:o + T, h] = p @ kv[:, 128:]
                if grad:
                    go = s.go[l, o:o + T, h].double()
                    dp = go @ kv[:, 128:].t()
                    dz = p * (dp - (p * dp).sum(-1, keepdim=True)) * s.scale
                    gq[l, o:o + T, h, :128] = dz @ kv[:, :128]
                    gq[l, o:o + T, h, 128:] = dz @ kr
                    gkv[l, o:o + T, h, :128] = dz.t() @ q[:, :128]
                    gkv[l, o:o + T, h, 128:] = p.t() @ go
                    gkr[l, o:o + T] += dz.t() @ q[:, 128:]
    return [gq, gkv, gkr] if grad else [out, lse]
