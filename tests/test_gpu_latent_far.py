"""Latent attention where single keys and far masks decide: weights that sit on one key at the edges of tiles, pages and pieces of long
sequences, gradients behind the 256th tile of keys."""
import numpy as np
import pytest
import torch

from helpers import ngc, status_value
from oracle import latent as ora
from test_gpu_latent import Replay, assert_within, bf16, f32, host, normal, random_pool, run_decode

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------ absorbed form

def piece_edges(lens, pieces):
    """Tiles (sequence, tile) that a piece of the line of 64-token tiles begins with, and the ones before them."""
    tiles = [(s, t) for s, n in enumerate(lens) for t in range(-(-n // 64))]
    used = max(1, min(pieces, len(tiles)))
    cuts = {len(tiles) * i // used for i in range(used)}
    return [tiles[g] for g in sorted(c + d for c in cuts for d in (-1, 0) if 0 <= c + d < len(tiles))]


@pytest.mark.parametrize("H,dc,dr,page,lens", [(16, 512, 64, 64, [9001]), (12, 128, 16, 32, [20000, 1, 64, 129]), (64, 256, 32, 32, [5000, 4999]),
                                               (128, 512, 64, 64, [3333, 65, 7000]), (16, 512, 64, 32, [700] * 40)])
def test_decode_finds_the_one_key_that_counts(H, dc, dr, page, lens):
    """Every head's weights sit on two keys of its own, which lie at the edges of tiles, pages and pieces and among them the first and last
    token: one of them lost, taken twice or taken from elsewhere is an error of half the output's size."""
    b = ngc()
    B = len(lens)
    pool = random_pool(1, B, page, -(-max(lens) // page), sum(-(-n // page) for n in lens) + 3, lens, 0, 50 + H, dc, dr)
    table = host(pool.page_table)
    rng = np.random.default_rng(H)
    edges = [set() for _ in lens]
    for s, t in piece_edges(lens, 148 // max(1, -(-H // 64))):
        edges[s] |= {64 * t, min(64 * t + 63, lens[s] - 1)}
    for s, n in enumerate(lens):
        edges[s] |= {x for x in (0, 31, 32, 63, 64, n - 1, n // 64 * 64 - 1, n // 64 * 64) if 0 <= x < n}
    rows = host(pool.rows).reshape(-1, dc + dr)
    ql, qr = normal((1, B, H, dc), 1), normal((1, B, H, dr), 2)
    q = np.concatenate([host(ql), host(qr)], -1)[0]
    for s in range(B):
        e = sorted(edges[s])
        at = rng.choice(e, (H, 2)) if s else np.array([[e[(2 * h) % len(e)], e[(2 * h + 1) % len(e)]] for h in range(H)])
        for h in range(H):
            for t in at[h]:                                                  # (a key of several heads belongs to the last of them)
                rows[table[s, 0, t // page] * page + t % page] = 12.0 * q[s, h] / np.linalg.norm(q[s, h])
    pool.rows.copy_(torch.as_tensor(rows).to(bf16).view(pool.rows.shape))
    # a heavy key's score is 12 |q| * scale = 18, the others' are normal with deviation 1.5 (1.8 with few channels: 4 are loud), some 7 at
    # most and exp(11) together
    scale = 1.5 / float(np.linalg.norm(q, axis=-1).mean())
    out, st = torch.zeros((1, B, H, dc), device="cuda"), b.new_status()
    b.ngc_latent_decode(pool, ql.cuda(), qr.cuda(), out, scale, ws=b.alloc_workspace(b.latent_decode_workspace_bytes(pool, H)), status=st)
    assert status_value(st) == 0
    want, bound = ora.decode(host(pool.rows), table, host(pool.lens), host(ql), host(qr), scale, 0)
    assert_within(out, want, bound)


@pytest.mark.parametrize("lens", [[1, 1, 300], [9001, 9001, 70], [70] * 150])
def test_scores_without_a_number(lens):
    """A rotary infinity in one key: plus infinity makes the head NaN; minus infinity takes the key out, and where it is the only key, leaves
    no score at all: NaN too.  Whole units and ones in many parts; the last sequence has none of it."""
    B, dc, dr, page = len(lens), 128, 16, 64
    pool = random_pool(1, B, page, -(-max(lens) // page), sum(-(-n // page) for n in lens) + 1, lens, 0, 71, dc, dr)
    clean, table = host(pool.rows), host(pool.page_table)
    for s in range(B - 1):
        t = lens[s] - 1
        pool.rows[0, table[s, 0, t // page], t % page, dc + 3] = float("inf")
    ql, qr, out, st = run_decode(pool, 8, 0.1)
    assert status_value(st) == 0
    out, up = out[0].cpu(), qr[0, :, :, 3].float() > 0
    for s in range(B - 1):
        assert bool(torch.isnan(out[s, up[s]]).all())
        assert bool((torch.isnan if lens[s] == 1 else torch.isfinite)(out[s, ~up[s]]).all())
    want, bound = ora.decode(clean, table[-1:], host(pool.lens)[-1:], host(ql)[:, -1:], host(qr)[:, -1:], 0.1, 0)
    assert_within(out[None, -1:], want, bound)


# ------------------------------------------------------------------ expanded form

def last_queries(r, n, rounds):
    """By the definition: out, grad_q of the last n queries, and what they alone give to the gradients of the last n keys (no earlier
    query sees those), each with its bound."""
    T, scale = r.lens[0], r.scale
    q, kv, kr, go = (host(x[0]).astype(np.float64) for x in (r.q, r.kv, r.kr, r.go))
    q, go = q[-n:, 0], go[-n:, 0]
    see = np.arange(T)[None, :] <= np.arange(T - n, T)[:, None]
    if rounds:
        fired, kept = r.hist[0][0][-1]
        assert fired <= T - n
        see[:, :fired] = False
        see[:, kept] = True
    k, v = np.concatenate([kv[:, 0, :128], kr], -1), kv[:, 0, 128:]
    z = np.where(see, scale * q @ k.T, -np.inf)
    p, lse = ora._softmax(z)
    dz_err = k.shape[1] * ora.U32 * scale * (np.abs(q) @ np.abs(k).T).max(-1, keepdims=True)
    e = 2 * dz_err + ora.EXP + T * ora.U32
    out = p @ v
    res = [(out, (ora.U16 + e) * (p @ np.abs(v)) + e * np.abs(out))]
    # the gradient from the call's own out and lse
    o, lse = host(r.out[0, -n:, 0]).astype(np.float64), host(r.lse[0, 0, -n:]).astype(np.float64)
    p = np.where(see, np.exp(np.where(see, z, 0.0) - lse[:, None]), 0.0)
    dz = scale * p * (go @ v.T - (go * o).sum(-1, keepdims=True))
    ez = dz_err + ora.EXP + 4 * ora.U32 * np.abs(lse)[:, None]
    ep = (ora.U16 + ez) * p
    edp = 128 * ora.U32 * (np.abs(go) @ np.abs(v).T + (np.abs(go) * np.abs(o)).sum(-1, keepdims=True))
    edz = (ora.U16 + ez) * np.abs(dz) + scale * p * edp * (1 + ez)
    f = T * ora.U32
    gq = dz @ k
    res.append((gq, (edz + f * np.abs(dz)) @ np.abs(k) + ora.U16 * np.abs(gq)))
    gk, bk = (dz.T @ q)[-n:], ((edz + f * np.abs(dz)).T @ np.abs(q))[-n:]
    gv, bv = (p.T @ go)[-n:], ((ep + f * p).T @ np.abs(go))[-n:]
    return res + [(x, y + ora.U16 * np.abs(x)) for x, y in ((gk[:, :128], bk[:, :128]), (gv, bv), (gk[:, 128:], bk[:, 128:]))]


@pytest.mark.parametrize("T,rounds", [(33500, [(0.5, 0.001), (0.9, 0.5)]), (33500, [(0.985, 0.3)]), (33011, None)])
def test_gradients_behind_the_plans_masks(T, rounds):
    """More than 256 tiles of keys: masks that are not planned ahead, in the forward pass, in the queries' walk by halves of tiles and in the
    keys' walk; nearly all keys gone, a third left, none gone."""
    r = Replay(1, 1, 1, 16, [T], 0, 83, rounds)
    r.forward(f32)
    r.backward()
    assert status_value(r.st) == 0
    n = 300
    got = [r.out[0, -n:, 0], r.grads[0][0, -n:, 0], r.grads[1][0, -n:, 0, :128], r.grads[1][0, -n:, 0, 128:], r.grads[2][0, -n:]]
    for name, g, (want, bound) in zip(("out", "grad q", "grad k", "grad v", "grad k_rope"), got, last_queries(r, n, rounds)):
        assert_within(g, want, bound, name)
