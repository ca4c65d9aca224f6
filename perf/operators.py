"""Cases that measure the drafted-token operators: attention for a tree of drafted tokens over the
pruned cache, verification of the drafts, the commit of the accepted rows, and the fork of a prefilled
prompt to its rollouts.

``run`` computes a case in plain torch operations (``own`` false) or through the library's entry points
(``own`` true); both take what ``prepare`` gives.  ``exact`` is the attention from its definition in 64
bits; the other operators move rows or decide on whole numbers and have no floating outputs of their own.
"""
from __future__ import annotations

import math
import types

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def listed():
    return [
        # one pending token of one rollout, called layer by layer: nothing but latency
        dict(name="tree_one_node", op="tree_attn", layers=1, batch=1, hq=12, hkv=2, d=128, dtype="bf16", t_lo=512, t_hi=512,
             nodes=1, shape="chain", ragged_nodes=False, page=0, lists=0, per_list=False),
        # a serving step of a model that calls its layers one by one: ragged rollouts, trees of up to 16 nodes
        dict(name="tree_layer_b64", op="tree_attn", layers=1, batch=64, hq=12, hkv=2, d=128, dtype="bf16", t_lo=1024, t_hi=4096,
             nodes=16, shape="tree", ragged_nodes=True, page=0, lists=0, per_list=False),
        # several layers in one call on the paged cache after uneven evictions: a length per list, odd node count, 7 heads a group
        dict(name="tree_paged_lists", op="tree_attn", layers=4, batch=16, hq=28, hkv=4, d=128, dtype="bf16", t_lo=1024, t_hi=8192,
             nodes=33, shape="tree", ragged_nodes=False, page=32, lists=1, per_list=True),
        # one very long cache under a large tree: the token axis is all the parallelism there is
        dict(name="tree_long", op="tree_attn", layers=2, batch=1, hq=12, hkv=2, d=128, dtype="bf16", t_lo=131072, t_hi=131072,
             nodes=64, shape="tree", ragged_nodes=False, page=0, lists=0, per_list=False),
        # the tiny fp32 workload with short chains
        dict(name="tree_fp32", op="tree_attn", layers=1, batch=4, hq=4, hkv=4, d=64, dtype="f32", t_lo=300, t_hi=512,
             nodes=8, shape="chain", ragged_nodes=False, page=0, lists=0, per_list=False),
        # a chain of four drafts for one rollout
        dict(name="verify_chain", op="verify", batch=1, nodes=5, vocab=32768, shape="chain", ragged_nodes=False, mode="draft"),
        # trees drawn from a draft model for a batch of rollouts, large vocabulary
        dict(name="verify_tree", op="verify", batch=64, nodes=17, vocab=131072, shape="tree", ragged_nodes=True, mode="draft"),
        # trees of the draft's likeliest tokens (no draft probabilities), odd vocabulary: rows that start on no 16-byte border
        dict(name="verify_point", op="verify", batch=48, nodes=33, vocab=50001, shape="tree", ragged_nodes=False, mode="point"),
        # the accepted rows of one rollout, all layers
        dict(name="commit_one", op="commit", layers=28, batch=1, hq=12, hkv=2, d=128, dtype="bf16", t_lo=700, t_hi=700, spare=16,
             nodes=8, accepted=4, page=0, lists=0, per_list=False),
        # a large batch on the paged cache, layers with lengths of their own
        dict(name="commit_paged", op="commit", layers=28, batch=256, hq=12, hkv=2, d=128, dtype="bf16", t_lo=200, t_hi=330, spare=16,
             nodes=16, accepted=7, page=32, lists=1, per_list=True),
        # one prompt to the eight rollouts of its group, paged
        dict(name="fork_pages", op="fork", layers=28, prompts=1, group=8, hq=12, hkv=2, d=128, dtype="bf16", t_lo=350, t_hi=350,
             spare=64, page=32, lists=1, per_list=False),
        # four prompts of about a thousand tokens to sixteen rollouts each
        dict(name="fork_prompts", op="fork", layers=28, prompts=4, group=16, hq=12, hkv=2, d=128, dtype="bf16", t_lo=900, t_hi=1100,
             spare=52, page=0, lists=0, per_list=False),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["tree_attn", "tree_attn", "verify", "commit", "fork"])
    if op == "verify":
        c = dict(op=op, batch=_log(rng, 1, 96), nodes=_log(rng, 1, 64), vocab=_log(rng, 1000, 150000), shape=rng.choice(["chain", "tree"]),
                 ragged_nodes=rng.random() < 0.5, mode=rng.choice(["draft", "point", "greedy"]))
        while c["batch"] * c["nodes"] * c["vocab"] > 64 * 17 * 131072:
            c["batch"] = max(1, c["batch"] // 2)
            c["vocab"] = max(1000, c["vocab"] * 3 // 4)
        return c
    hq, hkv = rng.choice([(12, 2), (28, 4), (4, 4), (16, 1), (6, 3), (40, 2)])
    layout = rng.choice(["contiguous", "paged"])
    dtype, d = ("bf16", 128) if layout == "paged" else rng.choice([("bf16", 128), ("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
    lists = rng.choice([0, 1, 2])
    c = dict(op=op, layers=rng.choice([1, 2, 3, 5]), hq=hq, hkv=hkv, d=d, dtype=dtype, page=rng.choice([32, 64]) if layout == "paged" else 0,
             lists=lists, per_list=lists != 0 and rng.random() < 0.5)
    row = 2 * d * (2 if dtype == "bf16" else 4)          # bytes of one token's K and V row
    if op == "tree_attn":
        t_hi = _log(rng, 1, 65536)
        c.update(batch=_log(rng, 1, 64), t_lo=rng.choice([t_hi, t_hi // 2, 0]), t_hi=t_hi, nodes=_log(rng, 1, 128), shape=rng.choice(["chain", "tree"]),
                 ragged_nodes=rng.random() < 0.5)
        flops = 4 * d * hq * c["layers"] * t_hi * c["nodes"] * (16 if dtype == "f32" else 1)
        while c["batch"] > 1 and c["batch"] * max(flops / 1e11, c["layers"] * hkv * t_hi * row / 4e8) > 1:
            c["batch"] //= 2
        while c["t_hi"] > 1 and c["batch"] * c["t_hi"] / t_hi * max(flops / 1e11, c["layers"] * hkv * t_hi * row / 4e8) > 1:
            c["t_hi"] //= 2
        c["t_lo"] = min(c["t_lo"], c["t_hi"])
        return c
    if op == "commit":
        t_hi = _log(rng, 1, 4096)
        nodes = _log(rng, 1, 128)
        c.update(batch=_log(rng, 1, 256), t_lo=t_hi // 2, t_hi=t_hi, spare=nodes + rng.randrange(40), nodes=nodes, accepted=rng.randint(1, nodes))
        while c["batch"] > 1 and c["batch"] * c["layers"] * hkv * (t_hi + c["spare"]) * row > 2e9:
            c["batch"] //= 2
        return c
    t_hi = _log(rng, 1, 8192)
    c.update(prompts=_log(rng, 1, 8), group=_log(rng, 2, 32), t_lo=t_hi // 2, t_hi=t_hi, spare=rng.randrange(100))
    while c["prompts"] * c["group"] * c["layers"] * hkv * (t_hi + c["spare"]) * row > 1.5e9:
        c["t_hi"] = t_hi = t_hi // 2
        c["t_lo"] = t_hi // 2
    return c


# ---------------------------------------------------------------- inputs, from the seed alone

def _spread(lo, hi, n):
    """n whole numbers from lo to hi, evenly spaced: the same sum whatever their order."""
    return [hi if n == 1 else lo + (hi - lo) * i // (n - 1) for i in range(n)]


def _lists(c):
    return 1 if c["lists"] == 0 else c["layers"] * (c["hkv"] if c["lists"] == 2 else 1)


def _batch(c):
    return c["batch"] if c["op"] != "fork" else c["prompts"] * c["group"]


def _nodes(c):
    return _spread(max(1, c["nodes"] // 2), c["nodes"], c["batch"]) if c.get("ragged_nodes") else [c["nodes"]] * c["batch"]


def _lens(c):
    """Cache lengths of the case, in some order: one per sequence, or one per (sequence, list); of a fork, those of the prompts."""
    per = _lists(c) if c["per_list"] else 1
    return _spread(c["t_lo"], c["t_hi"], (c["prompts"] if c["op"] == "fork" else c["batch"]) * per)


def _shuffled(values, g, shape):
    t = torch.tensor(values, dtype=torch.int32)
    return t[torch.randperm(len(values), generator=g)].reshape(shape).cuda()


def _tree(c, g, batch, nodes):
    """Parents [batch][nodes]: node 0 is the root, every parent comes before its children."""
    i = torch.arange(nodes)
    if c["shape"] == "chain":
        return (i - 1).expand(batch, nodes).contiguous().to(torch.int32).cuda()
    back = (torch.rand(batch, nodes, generator=g) * i.clamp(max=8)).long().clamp(max=7)
    return torch.where(i == 0, -1, (i - 1 - back).clamp(min=0)).to(torch.int32).cuda()


def _cache(c, s, g, gd):
    """K and V of every sequence with its spare rows, contiguous or in pages, and the cache lengths."""
    L, B, Hkv, d, dt = c["layers"], _batch(c), c["hkv"], c["d"], DTYPES[c["dtype"]]
    per = _lists(c) if c["per_list"] else 1
    cap = max(1, c["t_hi"] + c.get("spare", 0))
    pages = -(-cap // c["page"]) if c["page"] else 0
    cap = pages * c["page"] if pages else cap
    # random bits of normal numbers, a plane at a time
    s.k, s.v = (torch.empty((L, Hkv, B * cap, d), dtype=dt, device="cuda") for _ in range(2))
    for t in (s.k, s.v):
        t.normal_(generator=gd)
    s.k[:, :, :, :4] *= 4                                   # a few loud key channels, as trained models have
    lens = _shuffled(_lens(c), g, (-1, per))
    if c["op"] == "fork":
        full = torch.zeros((c["prompts"], c["group"], per), dtype=torch.int32, device="cuda")
        full[:, 0] = lens                                   # the first sequence of every group holds the prompt
        lens = full.reshape(B, per)
    s.lens = lens.contiguous() if c["per_list"] else lens.reshape(B).contiguous()
    s.cap = cap
    if pages:
        s.table = torch.stack([torch.randperm(pages, generator=g) for _ in range(B * _lists(c))]).reshape(B, _lists(c), pages).to(torch.int32).cuda()
        s.k, s.v = (t.reshape(L, Hkv, B * pages, c["page"], d) for t in (s.k, s.v))
    else:
        s.seq_off = (torch.arange(B + 1) * cap).cuda()


def _inputs(c, seed):
    g = torch.Generator().manual_seed(int(seed) * 7919 + 1)
    gd = torch.Generator(device="cuda").manual_seed(int(seed) * 104729 + 3)
    s = types.SimpleNamespace(case=c)
    B, N = _batch(c), c.get("nodes", 0)
    if c["op"] == "verify":
        V = c["vocab"]
        s.parent = _tree(c, g, B, N)
        s.n_nodes = _shuffled(_nodes(c), g, (B,)) if c["ragged_nodes"] else None
        z = torch.randn((B, N, V), generator=gd, device="cuda") * 3
        s.p = torch.softmax(z, -1)
        z += torch.randn((B, N, V), generator=gd, device="cuda") * 0.7
        q = torch.softmax(z, -1)
        del z
        up = s.parent.clamp(min=0).long()
        if c["mode"] == "draft":                            # every child an independent draw from its parent's draft row
            cdf = q.double().cumsum(-1)
            cdf = torch.gather(cdf, 1, up[:, :, None].expand(B, N, V)) if N > 1 else cdf
            u = torch.rand((B, N, 1), generator=gd, device="cuda", dtype=torch.float64) * cdf[:, :, -1:]
            s.tokens = torch.searchsorted(cdf, u, right=True).clamp(max=V - 1).reshape(B, N).to(torch.int32)
            s.q = q
        else:                                               # the r-th child of a node carries the draft's r-th likeliest token
            par = s.parent.cpu()
            rank = ((par[:, :, None] == par[:, None, :]) & (torch.arange(N)[None, :] < torch.arange(N)[:, None])).sum(-1).cuda()
            top = q.topk(int(rank.max()) + 1, -1).indices
            s.tokens = top[torch.arange(B, device="cuda")[:, None], up, rank].to(torch.int32)
            s.q = None
        s.tokens = s.tokens.contiguous()
        s.u = torch.rand((B, N), generator=gd, device="cuda")
        s.path = torch.empty((B, N), dtype=torch.int32, device="cuda")
        s.n_path = torch.empty((B,), dtype=torch.int32, device="cuda")
        s.next = torch.empty((B,), dtype=torch.int32, device="cuda")
        return s
    _cache(c, s, g, gd)
    L, Hq, Hkv, d, dt = c["layers"], c["hq"], c["hkv"], c["d"], DTYPES[c["dtype"]]
    if c["op"] == "fork":
        src = torch.arange(c["prompts"]).repeat_interleave(c["group"]) * c["group"]
        s.src_of = torch.where(src == torch.arange(B), -1, src).to(torch.int32).cuda()
        return s
    s.tk = torch.randn((L, B, Hkv, N, d), generator=gd, device="cuda").to(dt)
    s.tv = torch.randn((L, B, Hkv, N, d), generator=gd, device="cuda").to(dt)
    if c["op"] == "commit":
        n = c["accepted"]
        keep = torch.rand((B, N), generator=g)
        keep[:, 0] = -1                                     # the root is always on the path
        path = keep.argsort(-1)[:, :n].sort(-1).values
        s.path = torch.full((B, N), -1, dtype=torch.int32)
        s.path[:, :n] = path.to(torch.int32)
        s.path = s.path.cuda()
        s.n_path = torch.full((B,), n, dtype=torch.int32, device="cuda")
        s.lens0 = s.lens.clone()
        return s
    s.parent = _tree(c, g, B, N)
    s.n_nodes = _shuffled(_nodes(c), g, (B,)) if c["ragged_nodes"] else None
    s.q = torch.randn((L, B, Hq, N, d), generator=gd, device="cuda").to(dt)
    s.out = torch.zeros((L, B, Hq, N, d), dtype=dt, device="cuda")
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:
        from paper_2604_18002_b200 import binding as ngc
        s.status = ngc.new_status()
        if case["op"] != "verify":
            if case["page"]:
                s.cache = ngc.NgcPagedCache(s.k, s.v, s.table, s.lens, case["hq"], case["lists"])
            else:
                s.cache = ngc.NgcCache(s.k, s.v, s.seq_off, s.lens, case["hq"], s.cap, case["lists"] if case["per_list"] else 0)
        if case["op"] == "tree_attn":
            flat = s.cache.as_contiguous_desc() if case["page"] else s.cache
            s.ws = ngc.alloc_workspace(ngc.workspace_bytes(ngc.OP_TREE_ATTN, flat, n_max=case["nodes"]))
    return s


# ---------------------------------------------------------------- one pass

def run(state):
    op = state.case["op"]
    if own:
        return _OWN[op](state)
    return _PLAIN[op](state)


def _own_tree(s):
    from paper_2604_18002_b200 import binding as ngc
    call = ngc.ngc_tree_attn_paged if s.case["page"] else ngc.ngc_tree_attn
    call(s.cache, s.q, s.tk, s.tv, s.parent, s.out, n_nodes=s.n_nodes, ws=s.ws, status=s.status)
    return s.out


def _own_verify(s):
    from paper_2604_18002_b200 import binding as ngc
    ngc.ngc_verify_draft(s.tokens, s.parent, s.p, s.u, s.path, s.n_path, s.next, draft_probs=s.q, n_nodes=s.n_nodes,
                         greedy=int(s.case["mode"] == "greedy"), status=s.status)
    return [s.path, s.n_path, s.next]


def _own_commit(s):
    from paper_2604_18002_b200 import binding as ngc
    s.lens.copy_(s.lens0)                                   # back to the lengths before the drafts, then on with the accepted rows
    call = ngc.ngc_commit_draft_paged if s.case["page"] else ngc.ngc_commit_draft
    call(s.cache, s.tk, s.tv, s.path, s.n_path, status=s.status)
    return [s.k, s.v, s.lens]


def _own_fork(s):
    from paper_2604_18002_b200 import binding as ngc
    call = ngc.ngc_fork_pages if s.case["page"] else ngc.ngc_fork_kv
    call(s.cache, s.src_of, status=s.status)
    return [s.k, s.v, s.lens]


_OWN = dict(tree_attn=_own_tree, verify=_own_verify, commit=_own_commit, fork=_own_fork)


def _strip_rows(s, t):
    """Rows of the planes that hold tokens t [B or 1][T] of every strip: [L][Hkv][B][T]."""
    c = s.case
    L, Hkv, B = c["layers"], c["hkv"], _batch(c)
    b = torch.arange(B, device="cuda")
    if not c["page"]:
        return (s.seq_off[:B, None] + t).expand(L, Hkv, B, -1)
    l, h = torch.arange(L, device="cuda")[:, None, None], torch.arange(Hkv, device="cuda")[None, :, None]
    gi = (0 * l + 0 * h if c["lists"] == 0 else l + 0 * h if c["lists"] == 1 else l * Hkv + h).expand(L, Hkv, B)
    pages = s.table.shape[2]
    tt = t.expand(L, Hkv, B, -1)
    page = torch.gather(s.table[b, gi].long(), -1, (tt // c["page"]).clamp(max=pages - 1))
    return (b[:, None] * pages + page) * c["page"] + tt % c["page"]


def _strip_lens(s, lens):
    """Lengths [B] or [B][G] as [L][Hkv][B]."""
    c = s.case
    L, Hkv, B = c["layers"], c["hkv"], _batch(c)
    if lens.dim() == 1:
        return lens.long().expand(L, Hkv, B)
    per = lens.long().t().reshape(L, -1, B)                 # a list per layer, or per layer and head
    return per.expand(L, Hkv, B)


def _plain_tree(s):
    c = s.case
    L, B, Hq, Hkv, d, N = c["layers"], c["batch"], c["hq"], c["hkv"], c["d"], c["nodes"]
    g, T = Hq // Hkv, c["t_hi"]
    t = torch.arange(T, device="cuda")[None, :]
    at = (torch.arange(L * Hkv, device="cuda").reshape(L, Hkv, 1, 1), _strip_rows(s, t))
    live = t < _strip_lens(s, s.lens)[..., None]            # [L][Hkv][B][T]
    k = s.k.reshape(L * Hkv, -1, d)[at].float()
    v = torch.where(live[..., None], s.v.reshape(L * Hkv, -1, d)[at].float(), 0.0)
    # who is an ancestor of whom (or itself): repeated squaring of parent links
    seen = torch.eye(N, device="cuda") + (s.parent[:, :, None] == torch.arange(N, device="cuda"))
    for _ in range(max(1, (N - 1).bit_length())):
        seen = ((seen @ seen) > 0).float()
    nodes = s.n_nodes if s.n_nodes is not None else torch.full((B,), N, device="cuda")
    alive = torch.arange(N, device="cuda") < nodes[:, None]                     # [B][N]
    see = (seen > 0) & alive[:, None, :]
    q = s.q.float().reshape(L, B, Hkv, g * N, d).transpose(1, 2)                # [L][Hkv][B][g N][d]
    tk, tv = s.tk.float().transpose(1, 2), s.tv.float().transpose(1, 2)
    tv = torch.where(alive[:, :, None], tv, 0.0)
    scale = 1.0 / math.sqrt(d)
    z = torch.cat([torch.where(live[:, :, :, None, :], (q @ k.transpose(-1, -2)) * scale, -math.inf),
                   torch.where(see.repeat(1, g, 1), (q @ tk.transpose(-1, -2)) * scale, -math.inf)], -1)
    z = torch.exp(z - z.amax(-1, keepdim=True).clamp(min=-1e30))
    o = (z[..., :T] @ v + z[..., T:] @ tv) / z.sum(-1, keepdim=True)
    o = o.reshape(L, Hkv, B, g, N, d).permute(0, 2, 1, 3, 4, 5).reshape(L, B, Hq, N, d)
    s.out.copy_(torch.where(alive[:, None, :, None], o, 0.0))
    return s.out


def _plain_verify(s):
    c = s.case
    B, N, V = c["batch"], c["nodes"], c["vocab"]
    rows = torch.arange(B, device="cuda")
    nodes = s.n_nodes.long() if s.n_nodes is not None else torch.full((B,), N, device="cuda")
    par, tok = s.parent.long(), s.tokens.long()
    cur = torch.zeros(B, dtype=torch.long, device="cuda")
    n_path = torch.ones(B, dtype=torch.long, device="cuda")
    s.path.fill_(-1)
    s.path[:, 0] = 0
    tried = torch.zeros((B, V), dtype=torch.bool, device="cuda")                # tokens refused at the current node
    cut = torch.zeros(B, dtype=torch.float64, device="cuda")                    # what the refusals took off, in draft rows
    mass = torch.ones(B, dtype=torch.float64, device="cuda")
    if c["mode"] == "greedy":
        best = torch.where(s.p == s.p.amax(-1, keepdim=True), torch.arange(V, device="cuda"), V).amin(-1)
    for i in range(1, N):
        mine = (par[:, i] == cur) & (i < nodes)
        x, u = tok[:, i], s.u[:, i].double()
        p = s.p[rows, cur, x].double()
        if c["mode"] == "greedy":
            ok = mine & (best[rows, cur] == x)
        elif c["mode"] == "draft":
            q = s.q[rows, cur, x].double()
            ok = mine & (u * q * mass < p - cut * q)
            less = cut + mass
            rest = (s.p[rows, cur].double() - less[:, None] * s.q[rows, cur].double()).clamp(min=0).sum(-1)
            left = mine & ~ok & (rest > 0)                  # a residual without mass leaves the one before
            cut, mass = torch.where(left, less, cut), torch.where(left, rest, mass)
        else:
            p = torch.where(tried[rows, x], 0.0, p)
            ok = mine & (u * mass < p)
            left = mine & ~ok & (mass - p > 0)
            mass = torch.where(left, mass - p, mass)
            tried[rows, x] |= left
        s.path[rows, n_path.clamp(max=N - 1)] = torch.where(ok, i, s.path[rows, n_path.clamp(max=N - 1)]).to(torch.int32)
        n_path = n_path + ok
        cur = torch.where(ok, i, cur)
        cut, mass = torch.where(ok, 0.0, cut), torch.where(ok, 1.0, mass)
        tried &= ~ok[:, None]
    if c["mode"] == "greedy":
        nxt = best[rows, cur]
    else:
        w = s.p[rows, cur].double()
        if c["mode"] == "draft":
            w = (w - cut[:, None] * s.q[rows, cur].double()).clamp(min=0)
        else:
            w = torch.where(tried, 0.0, w)
        cdf = w.cumsum(-1)
        nxt = torch.searchsorted(cdf, s.u[:, :1].double() * cdf[:, -1:], right=True)[:, 0].clamp(max=V - 1)
    s.n_path.copy_(n_path)
    s.next.copy_(nxt)
    return [s.path, s.n_path, s.next]


def _plain_commit(s):
    c = s.case
    L, B, Hkv, d, n = c["layers"], c["batch"], c["hkv"], c["d"], c["accepted"]
    s.lens.copy_(s.lens0)
    t = _strip_lens(s, s.lens)[..., None] + torch.arange(n, device="cuda")      # [L][Hkv][B][n]
    if c["page"]:
        l, h = torch.arange(L, device="cuda")[:, None, None], torch.arange(Hkv, device="cuda")[None, :, None]
        b = torch.arange(B, device="cuda")
        gi = (0 * l + 0 * h if c["lists"] == 0 else l + 0 * h if c["lists"] == 1 else l * Hkv + h).expand(L, Hkv, B)
        at = (b[:, None] * s.table.shape[2] + torch.gather(s.table[b, gi].long(), -1, t // c["page"])) * c["page"] + t % c["page"]
    else:
        at = s.seq_off[:B, None] + t
    plane = torch.arange(L * Hkv, device="cuda").reshape(L, Hkv, 1, 1)
    node = s.path[:, :n].long()[None, :, None, :, None].expand(L, B, Hkv, n, d)
    for dst, src in ((s.k, s.tk), (s.v, s.tv)):
        dst.view(L * Hkv, -1, d)[plane, at] = torch.gather(src, 3, node).transpose(1, 2)
    s.lens += s.n_path if s.lens.dim() == 1 else s.n_path[:, None]
    return [s.k, s.v, s.lens]


def _plain_fork(s):
    c = s.case
    L, Hkv, B, d, T = c["layers"], c["hkv"], _batch(c), c["d"], c["t_hi"]
    src = torch.where(s.src_of < 0, torch.arange(B, device="cuda"), s.src_of.long())
    rows = _strip_rows(s, torch.arange(T, device="cuda")[None, :])              # [L][Hkv][B][T]
    move = (torch.arange(T, device="cuda") < _strip_lens(s, s.lens[src])[..., None]) & (s.src_of >= 0)[:, None]
    plane = torch.arange(L * Hkv, device="cuda").reshape(L, Hkv, 1, 1).expand(L, Hkv, B, T)[move]
    to, of = rows[move], rows[:, :, src][move]
    for t in (s.k, s.v):
        flat = t.view(L * Hkv, -1, d)
        flat[plane, to] = flat[plane, of]
    s.lens.copy_(s.lens[src])
    return [s.k, s.v, s.lens]


_PLAIN = dict(tree_attn=_plain_tree, verify=_plain_verify, commit=_plain_commit, fork=_plain_fork)


# ---------------------------------------------------------------- what a pass cannot do without

def work(case):
    c = case
    if c["op"] == "verify":
        # the row of the node at which the walk ends (and its draft row, where there is one), once
        n = c["batch"] * c["vocab"]
        return {"bytes": n * 4 * (2 if c["mode"] == "draft" else 1) + 16 * c["batch"] * c["nodes"], "flops": n * (4 if c["mode"] == "draft" else 1)}
    L, Hq, Hkv, d, B = c["layers"], c["hq"], c["hkv"], c["d"], _batch(c)
    e = 2 if c["dtype"] == "bf16" else 4
    planes = L * Hkv
    total = sum(_lens(c)) / (_lists(c) if c["per_list"] else 1)                 # tokens per plane, summed over the sequences
    if c["op"] == "commit":
        return {"bytes": 2 * 2 * planes * B * c["accepted"] * d * e, "flops": 0}
    if c["op"] == "fork":
        return {"bytes": 2 * planes * total * d * e * c["group"], "flops": 0}   # read once, written to the group - 1 others
    nodes = sum(_nodes(c))
    io = 2 * L * Hq * nodes * d * e + 2 * planes * nodes * d * e
    return {"bytes": 2 * planes * total * d * e + io, "flops": 4 * d * L * Hq * (total * nodes / B + nodes)}


# ---------------------------------------------------------------- the attention from its definition, in 64 bits

def exact(case, seed):
    c = case
    if c["op"] != "tree_attn":
        return None
    s = _inputs(c, seed)
    L, B, Hq, Hkv, d, N = c["layers"], c["batch"], c["hq"], c["hkv"], c["d"], c["nodes"]
    if L * B * Hkv > 4096:
        return None
    g = Hq // Hkv
    out = torch.zeros((L, B, Hq, N, d), dtype=torch.float64, device="cuda")
    lens, parent = s.lens.cpu().numpy(), s.parent.cpu().numpy()
    nodes = [N] * B if s.n_nodes is None else s.n_nodes.cpu().tolist()
    for b in range(B):
        n = int(nodes[b])
        mask = torch.zeros((n, n), dtype=torch.bool)
        for i in range(n):
            j = i
            while j >= 0:
                mask[i, j] = True
                j = int(parent[b, j])
        mask = mask.cuda()
        for l in range(L):
            for h in range(Hkv):
                gi = (0, l, l * Hkv + h)[c["lists"]]
                T = int(lens[b, gi]) if lens.ndim == 2 else int(lens[b])
                if c["page"]:
                    need = s.table[b, gi, : -(-T // c["page"])].long() + b * s.table.shape[2]
                    k, v = (x[l, h][need].reshape(-1, d)[:T].double() for x in (s.k, s.v))
                else:
                    o = b * s.cap
                    k, v = (x[l, h, o: o + T].double() for x in (s.k, s.v))
                k = torch.cat([k, s.tk[l, b, h, :n].double()])
                v = torch.cat([v, s.tv[l, b, h, :n].double()])
                q = s.q[l, b, h * g: h * g + g, :n].double()
                z = torch.einsum("hnd,td->hnt", q, k) / math.sqrt(d)
                z[:, :, T:].masked_fill_(~mask, -math.inf)
                out[l, b, h * g: h * g + g, :n] = torch.einsum("hnt,td->hnd", torch.softmax(z, -1), v)
    return out
