"""Plain implementations of the latent-attention calls, in 64 bits and written from their definitions: the page pool's books
step by step, attention over a pool, and attention of a whole sequence under its history of evictions with its gradient.

Beside every result stands a bound on what a correct kernel may be off by: each rounding to bf16 is off by at most half a step
(2**-8 of the value), an fp32 sum of n products by n * 2**-24 of the sum of their magnitudes, and the relative error of an
exponential is the absolute error of its argument.
"""
from __future__ import annotations

import numpy as np

U16 = 2.0 ** -8        # half a step of bf16
U32 = 2.0 ** -24
EXP = 2.0 ** -21       # fp32 exponential, its argument's scaling and the row sum's rounding, as a part of the value

OK, BAD_COUNTS, BAD_KEPT, STRIP_FULL, BAD_PAGE, POOL_FULL = 0, 1, 3, 4, 11, 12


def pool_update(table, used, lens, page, n_new, n_slots, kept=None, budget=None):
    """New (table, used, lens, slots, first) and the set of problems met (the library reports the first it meets)."""
    table, used, lens = table.copy(), used.copy(), lens.copy()
    B, G, cap = table.shape
    n_pages = used.shape[1]
    first = np.concatenate([[0], np.minimum(np.cumsum(np.maximum(n_new, 0).astype(np.int64)), 2 ** 30 - 1)]).astype(np.int32)
    slots = np.full((G, n_slots), -1, np.int32)
    problems = set()
    for g in range(G):
        grows = []
        for b in range(B):
            n, keep = int(n_new[b]), -1 if kept is None else int(budget[b])
            length = int(lens[b, g])
            if (not 0 <= length <= cap * page or n < -1 or n > max(n_slots - int(first[b]), 0) or keep < -1
                    or (kept is not None and keep > kept.shape[2])):
                problems.add(BAD_COUNTS)
                continue
            have = -(-length // page)
            row = [int(x) for x in table[b, g, :have]]
            if (keep >= 0 or n < 0) and any(not 0 <= x < n_pages for x in row):
                problems.add(BAD_PAGE)
                continue
            if keep >= 0:
                units = [int(x) for x in kept[b, g, :keep]]
                if any(not 0 <= u < have for u in units) or any(y <= x for x, y in zip(units, units[1:])):
                    problems.add(BAD_KEPT)
                    continue
            if keep >= 0 or n < 0:
                for x in row:
                    used[g, x] = 0
                tokens = 0
                if n < 0:
                    row = []
                else:
                    tokens = sum(min(page, length - u * page) for u in units)
                    row = [row[u] for u in units]
                for x in row:
                    used[g, x] = 1
                table[b, g, :have] = -1
                table[b, g, :len(row)] = row
                length = tokens
                lens[b, g] = length
            n = max(n, 0)
            if n > cap * page - length:
                problems.add(STRIP_FULL)
            elif n > 0 and length % page and not 0 <= table[b, g, length // page] < n_pages:
                problems.add(BAD_PAGE)
            else:
                grows.append((b, length, n))
        free = [x for x in range(n_pages) if used[g, x] == 0]
        at = 0
        for b, length, n in grows:
            have, need = -(-length // page), -(-(length + n) // page)
            if need - have > len(free) - at:                     # (those after it that need less may fit)
                problems.add(POOL_FULL)
                continue
            at += need - have
            for j in range(have, need):
                x = free[at - need + j]
                table[b, g, j] = x
                used[g, x] = 1
            for i in range(n):
                pos = length + i
                slots[g, first[b] + i] = table[b, g, pos // page] * page + pos % page
            lens[b, g] = length + n
    return table, used, lens, slots, first, problems


def _softmax(z):
    m = z.max(-1, keepdims=True)
    p = np.exp(z - np.where(np.isfinite(m), m, 0.0))
    total = p.sum(-1, keepdims=True)
    with np.errstate(divide="ignore"):
        lse = (np.where(np.isfinite(m), m, 0.0) + np.log(total))[..., 0]
    return np.where(total > 0, p / np.where(total > 0, total, 1.0), 0.0), lse


def _score_error(q, k, scale):
    """Bound on the error of every query's scores: the largest over its keys."""
    n = q.shape[-1]
    return n * U32 * scale * (np.abs(q) @ np.abs(k).T).max(-1, keepdims=True) if len(k) else np.zeros((len(q), 1))


def decode(rows, table, lens, ql, qr, scale, lists, bf16_out=False):
    """Absorbed form: rows [L][n_pages][page][dc + dr], ql [L][B][H][dc], qr [L][B][H][dr] -> (out, bound) [L][B][H][dc]."""
    L, B, H, dc = ql.shape
    page = rows.shape[2]
    out, bound = np.zeros(ql.shape), np.zeros(ql.shape)
    for l in range(L):
        for b in range(B):
            T = int(lens[b, l if lists else 0])
            x = np.stack([rows[l, table[b, l if lists else 0, t // page], t % page] for t in range(T)]).astype(np.float64) if T else np.zeros((0, rows.shape[3]))
            if T == 0:
                continue
            q = np.concatenate([ql[l, b], qr[l, b]], -1).astype(np.float64)
            p, _ = _softmax(scale * q @ x.T)
            v = x[:, :dc]
            out[l, b] = p @ v
            size = p @ np.abs(v)
            e = 2 * _score_error(q, x, scale) + EXP + T * U32
            bound[l, b] = (U16 + e) * size + e * np.abs(out[l, b]) + (U16 if bf16_out else 0) * np.abs(out[l, b])
    return out, bound


def visible(T, rounds):
    """[T][T] truth table of a sequence of T tokens, by walking through its life: ``rounds`` is a list of (sequence length when
    the round fired, positions kept)."""
    see = np.zeros((T, T), bool)
    cache = []
    fired = list(rounds)
    for t in range(T):
        while fired and fired[0][0] <= t:
            keep = set(int(x) for x in fired.pop(0)[1])
            cache = [x for x in cache if x in keep]
        cache.append(t)
        see[t, cache] = True
    return see


def replay(q, kv, kr, see, scale, bf16_out=False):
    """Expanded form of one sequence: q [T][H][128 + dr], kv [T][H][256], kr [T][dr] -> out [T][H][128], lse [H][T] and their bounds."""
    T, H, _ = q.shape
    out, lse, ob, lb = np.zeros((T, H, 128)), np.zeros((H, T)), np.zeros((T, H, 128)), np.zeros((H, T))
    for h in range(H):
        k = np.concatenate([kv[:, h, :128], kr], -1).astype(np.float64)
        v = kv[:, h, 128:].astype(np.float64)
        qh = q[:, h].astype(np.float64)
        p, lse[h] = _softmax(np.where(see, scale * qh @ k.T, -np.inf))
        out[:, h] = p @ v
        dz = _score_error(qh, k, scale)
        e = 2 * dz + EXP + T * U32
        ob[:, h] = (U16 + e) * (p @ np.abs(v)) + e * np.abs(out[:, h]) + (U16 if bf16_out else 0) * np.abs(out[:, h])
        with np.errstate(invalid="ignore"):
            lb[h] = dz[:, 0] + EXP + T * U32 + 4 * U32 * np.where(np.isfinite(lse[h]), np.abs(lse[h]), 0.0)
    return out, lse, ob, lb


def replay_grad(q, kv, kr, see, scale, out, lse, go):
    """Gradient by the formula, from a forward call's out and lse -> [(value, bound)] of q, kv and kr."""
    T, H, width = q.shape
    gq, gkv, gkr = np.zeros(q.shape), np.zeros(kv.shape), np.zeros(kr.shape)
    bq, bkv, bkr = np.zeros(q.shape), np.zeros(kv.shape), np.zeros(kr.shape)
    for h in range(H):
        k = np.concatenate([kv[:, h, :128], kr], -1).astype(np.float64)
        v, qh, g = kv[:, h, 128:].astype(np.float64), q[:, h].astype(np.float64), go[:, h].astype(np.float64)
        o = out[:, h].astype(np.float64)
        with np.errstate(invalid="ignore", over="ignore"):
            p = np.where(see, np.exp(np.where(see, scale * qh @ k.T, 0.0) - np.where(np.isfinite(lse[h]), lse[h], 0.0)[:, None]), 0.0)
        dz = scale * p * (g @ v.T - (g * o).sum(-1, keepdims=True))
        # what P and dz may be off by
        ez = _score_error(qh, k, scale) + EXP + 4 * U32 * np.abs(np.where(np.isfinite(lse[h]), lse[h], 0.0))[:, None]
        ep = (U16 + ez) * p
        e_dp = 128 * U32 * (np.abs(g) @ np.abs(v).T + (np.abs(g) * np.abs(o)).sum(-1, keepdims=True))
        edz = (U16 + ez) * np.abs(dz) + scale * p * e_dp * (1 + ez)
        f = T * U32                                                # the sum over tokens
        gq[:, h] = dz @ k
        bq[:, h] = (edz + f * np.abs(dz)) @ np.abs(k) + U16 * np.abs(gq[:, h])
        dk, bk = dz.T @ qh, (edz + f * np.abs(dz)).T @ np.abs(qh)
        gkv[:, h, :128], bkv[:, h, :128] = dk[:, :128], bk[:, :128] + U16 * np.abs(dk[:, :128])
        gkv[:, h, 128:] = p.T @ g
        bkv[:, h, 128:] = (ep + f * p).T @ np.abs(g) + U16 * np.abs(gkv[:, h, 128:])
        gkr += dk[:, 128:]
        bkr += bk[:, 128:] + H * U32 * np.abs(dk[:, 128:])
    return (gq, bq), (gkv, bkv), (gkr, bkr + U16 * np.abs(gkr))
