"""CPU oracle of the drafted-token calls, in numpy and float64, written from their definitions: attention
for a tree of drafted tokens over a cache, verification of the tree against the target's probabilities, the
append of the accepted rows and the fork of a sequence to others.

Bf16 arrays come as uint16 bit patterns (``synth.to_numpy``).  Nothing here looks at the CUDA code: paths are
followed link by link, residuals are formed one rejection at a time, rows are copied one by one."""
from __future__ import annotations

import numpy as np

from . import lists_G
from paper_2604_18002_b200.synth import as_f64


def ancestors(parent, i):
    """Node i and its ancestors, root last; None for a link that is none."""
    out = [int(i)]
    while out[-1] != 0:
        up = int(parent[out[-1]])
        if not 0 <= up < out[-1]:
            return None
        out.append(up)
    return out if int(parent[0]) == -1 else None


def tree_ok(parent, n, N):
    return 0 <= n <= N and all(ancestors(parent, i) is not None for i in range(n))


def _list(lists, l, h, Hkv):
    return (0, l, l * Hkv + h)[lists]


def strip_len(lens, lens_lists, b, l, h, Hkv):
    return int(lens[b]) if lens_lists == 0 else int(lens[b, _list(lens_lists, l, h, Hkv)])


def tree_attn(k, v, seq_off, lens, q, tk, tv, parent, n_nodes=None, scale=None, lens_lists=0, fill=0.0):
    """[L][B][Hq][N][d] float64; rows of nodes beyond a tree, and of refused trees, hold ``fill``."""
    L, B, Hq, N, d = q.shape
    Hkv = tk.shape[2]
    g = Hq // Hkv
    scale = 1.0 / np.sqrt(d) if scale is None else scale
    out = np.full(q.shape, fill, np.float64)
    for b in range(B):
        n = N if n_nodes is None else int(n_nodes[b])
        if not tree_ok(parent[b], n, N):
            continue
        for l in range(L):
            for h in range(Hkv):
                T, o = strip_len(lens, lens_lists, b, l, h, Hkv), int(seq_off[b])
                if not 0 <= T <= int(seq_off[b + 1]) - o:
                    continue
                kc, vc = as_f64(k[l, h, o:o + T]), as_f64(v[l, h, o:o + T])
                kt, vt = as_f64(tk[l, b, h]), as_f64(tv[l, b, h])
                for i in range(n):
                    a = ancestors(parent[b], i)
                    kk, vv = np.concatenate([kc, kt[a]]), np.concatenate([vc, vt[a]])
                    with np.errstate(all="ignore"):
                        for hq in range(h * g, h * g + g):
                            z = kk @ as_f64(q[l, b, hq, i]) * scale
                            w = np.exp(z - z.max())
                            out[l, b, hq, i] = (w[:, None] * vv).sum(0) / w.sum()
    return out


def verify_draft(tokens, parent, target, uniforms, draft=None, n_nodes=None, greedy=False):
    """(path [B][N], n_path [B], next_token [B], status [B]: 0 ok, 8 bad tree, 9 bad probabilities)."""
    B, N, V = target.shape
    path, n_path = np.full((B, N), -1, np.int32), np.zeros(B, np.int32)
    nxt, status = np.full(B, -1, np.int32), np.zeros(B, np.int32)
    for b in range(B):
        n = N if n_nodes is None else int(n_nodes[b])
        if not tree_ok(parent[b], n, N) or any(not 0 <= int(tokens[b, i]) < V for i in range(1, n)):
            status[b] = 8
            continue
        if n == 0:
            continue
        walk, cur = [0], 0
        while True:
            w, mass = target[b, cur].astype(np.float64), 1.0
            q = None if draft is None else draft[b, cur].astype(np.float64)
            if not greedy:
                w[w < 0] = 0.0
            if greedy and np.isnan(w).any():
                status[b] = 9
                break
            step = None
            for i in [j for j in range(1, n) if int(parent[b, j]) == cur]:
                x = int(tokens[b, i])
                if greedy:
                    ok = x == int(np.argmax(w))
                else:
                    if not all(0 <= float(r[b, cur, x]) < np.inf for r in (target, draft) if r is not None):
                        status[b] = 9
                        break
                    u = float(uniforms[b, i])
                    ok = u * mass < w[x] if q is None else u * q[x] * mass < w[x]
                if ok:
                    step = i
                    break
                if greedy:
                    continue
                if q is None:
                    if mass - w[x] > 0:
                        mass, w = mass - w[x], w.copy()
                        w[x] = 0.0
                else:
                    rest = w - mass * q
                    rest[rest < 0] = 0.0
                    total = rest.sum()
                    if not np.isfinite(total):
                        status[b] = 9
                        break
                    if total > 0:
                        w, mass = rest, total
            if step is None or status[b]:
                break
            cur = step
            walk.append(step)
        if status[b]:
            continue
        if greedy:
            nxt[b] = int(np.argmax(w))
        else:
            total = w.sum()
            if not (np.isfinite(total) and total > 0):
                status[b] = 9
                continue
            over = np.nonzero(np.cumsum(w) > float(uniforms[b, 0]) * total)[0]
            nxt[b] = over[0] if over.size else np.nonzero(w > 0)[0][-1]
        n_path[b] = len(walk)
        path[b, :len(walk)] = walk
    return path, n_path, nxt, status


def commit_draft(k, v, seq_off, lens, tk, tv, path, n_path, lens_lists=0):
    """Copies of (k, v, lens) after the append, and a status per sequence (0, 4 strip full, 8 bad path)."""
    k, v, lens = k.copy(), v.copy(), lens.copy()
    L, B, Hkv, N, _ = tk.shape
    status = np.zeros(B, np.int32)
    for b in range(B):
        n = int(n_path[b])
        p = [int(x) for x in path[b, :max(0, min(n, N))]]
        if not 0 <= n <= N or any(not 0 <= x < N for x in p) or any(y <= x for x, y in zip(p, p[1:])):
            status[b] = 8
            continue
        cap = int(seq_off[b + 1] - seq_off[b])
        at = {(l, h): strip_len(lens, lens_lists, b, l, h, Hkv) for l in range(L) for h in range(Hkv)}
        if any(t < 0 or t + n > cap for t in at.values()):
            status[b] = 4
            continue
        for (l, h), t in at.items():
            for j, x in enumerate(p):
                k[l, h, int(seq_off[b]) + t + j] = tk[l, b, h, x]
                v[l, h, int(seq_off[b]) + t + j] = tv[l, b, h, x]
        lens[b] += n
    return k, v, lens, status


def fork(k, v, seq_off, lens, src_of, lens_lists=0):
    """Copies of (k, v, lens) after the fork, and a status per sequence (0, 1 bad length, 4 too small, 10 bad source)."""
    k2, v2, lens2 = k.copy(), v.copy(), lens.copy()
    L, Hkv = k.shape[:2]
    B = len(src_of)
    status = np.zeros(B, np.int32)
    cap = [int(seq_off[b + 1] - seq_off[b]) for b in range(B)]
    for b in range(B):
        s = int(src_of[b])
        if s == -1 or s == b:
            continue
        if not 0 <= s < B or int(src_of[s]) not in (-1, s):
            status[b] = 10
            continue
        lens_s = [int(x) for x in np.atleast_1d(lens[s])]
        if any(not 0 <= t <= cap[s] for t in lens_s):
            status[b] = 1
            continue
        if max(lens_s) > cap[b]:
            status[b] = 4
            continue
        for l in range(L):
            for h in range(Hkv):
                t = strip_len(lens, lens_lists, s, l, h, Hkv)
                for a2, a in ((k2, k), (v2, v)):
                    a2[l, h, int(seq_off[b]):int(seq_off[b]) + t] = a[l, h, int(seq_off[s]):int(seq_off[s]) + t]
        lens2[b] = lens[s]
    return k2, v2, lens2, status


__all__ = ["ancestors", "tree_ok", "tree_attn", "verify_draft", "commit_draft", "fork", "lists_G"]
