"""Drafted-token calls on the GPU against the CPU oracle: tree attention (contiguous and paged), verification,
commit and fork; their refusals; and a run of them together."""
import numpy as np
import pytest
import torch

import oracle
from helpers import ngc, status_value
from oracle import draft
from paper_2604_18002_b200 import synth

pytestmark = pytest.mark.gpu

bf16, f32 = torch.bfloat16, torch.float32


def trees(B, N, kind, seed):
    rng = np.random.default_rng(seed)
    p = np.full((B, N), -1, np.int32)
    for i in range(1, N):
        if kind == "chain":
            p[:, i] = i - 1
        elif kind == "star":
            p[:, i] = 0
        else:
            p[:, i] = [rng.integers(max(0, i - 9), i) for _ in range(B)]
    return p


def case(dtype, d, Hq, Hkv, L, lens, N, kind="tree", seed=0, capacity=None, n_nodes=None):
    B = len(lens)
    c = synth.make_cache(L, B, Hq, Hkv, d, dtype, lens, capacity=capacity or max(max(lens), 1), seed=seed, outlier_channels=4)
    q, tk, tv = (synth.normal((L, B, H, N, d), seed + s, dtype) for H, s in ((Hq, 2), (Hkv, 3), (Hkv, 4)))
    return c, q, tk, tv, trees(B, N, kind, seed), None if n_nodes is None else np.asarray(n_nodes, np.int32)


def bound(c, q, tk, tv, parent, n_nodes, ref, lens_lists=0, out_bf16=False, scale=None):
    """How far a row may be off, element by element.  With weights w (sum 1) the output is sum w v.  A score is a dot
    product of d terms in fp32, so it is off by at most d 2^-24 sum |q k| scale =: ez, a weight by a factor
    1 + ez (+ 2^-22 of the exponential) above and below the line, hence 2 (ez + 2^-22) A in all, A = sum w |v|; the fp32
    sums over T keys add T 2^-24 A twice; on bf16 caches every weight is rounded once (2^-8 A); a bf16 output is
    rounded once (2^-8 |o|)."""
    f = synth.as_f64
    args = (f(synth.to_numpy(c.k)), np.abs(f(synth.to_numpy(c.v))), c.seq_off.numpy(), c.lens.numpy(), f(synth.to_numpy(q)),
            f(synth.to_numpy(tk)), np.abs(f(synth.to_numpy(tv))), parent, n_nodes)
    A = draft.tree_attn(*args, scale=scale, lens_lists=lens_lists)         # (the weights are those of the call's own scale)
    L, B, Hq, N, d = q.shape
    aq, ak, at = np.abs(args[4]), np.abs(args[0]), np.abs(args[5])
    g, so, most = Hq // at.shape[2], args[2], 0.0
    for b in range(B):
        for l in range(L):
            for h in range(at.shape[2]):
                rows = aq[l, b, h * g:h * g + g].reshape(-1, d)
                T = min(max(0, draft.strip_len(args[3], lens_lists, b, l, h, at.shape[2])), int(so[b + 1] - so[b]))
                for kk in (ak[l, h, so[b]:so[b] + T], at[l, b, h]):
                    most = max(most, float((rows @ kk.T).max()) if len(kk) else 0.0)
    ez = d * 2.0 ** -24 * most * (1 / np.sqrt(d) if scale is None else scale)
    T = int(np.max(args[3])) + q.shape[3]
    b = (2 * (ez + 2.0 ** -22) + 2 * T * 2.0 ** -24 + (2.0 ** -8 if c.k.dtype == bf16 else 0)) * A + 1e-30
    return b + (2.0 ** -8 * np.abs(ref) if out_bf16 else 0)


def run_tree(c, q, tk, tv, parent, n_nodes, out_dtype=None, lens=None, lens_lists=0, fill=-7.0, max_len=None, **kw):
    b = ngc()
    out = torch.full(q.shape, fill, dtype=out_dtype or f32, device="cuda")
    cap = int((c.seq_off[1:] - c.seq_off[:-1]).max())
    dc = b.NgcCache(c.k.cuda(), c.v.cuda(), c.seq_off.cuda(), (c.lens if lens is None else lens).cuda(), c.Hq, max_len or cap, lens_lists)
    ws = b.alloc_workspace(b.workspace_bytes(b.OP_TREE_ATTN, dc, n_max=q.shape[3]))
    st = b.new_status()
    b.ngc_tree_attn(dc, q.cuda(), tk.cuda(), tv.cuda(), torch.as_tensor(parent).cuda(), out,
                    None if n_nodes is None else torch.as_tensor(n_nodes).cuda(), ws=ws, status=st, **kw)
    torch.cuda.synchronize()
    return out, status_value(st)


def check_tree(c, q, tk, tv, parent, n_nodes, out_dtype=None, lens_lists=0, **kw):
    out, st = run_tree(c, q, tk, tv, parent, n_nodes, out_dtype, lens_lists=lens_lists, **kw)
    assert st == 0
    n = [synth.to_numpy(x) for x in (q, tk, tv)]
    ref = draft.tree_attn(synth.to_numpy(c.k), synth.to_numpy(c.v), c.seq_off.numpy(), c.lens.numpy(), *n, parent, n_nodes,
                          lens_lists=lens_lists, fill=-7.0, scale=kw.get("scale"))
    lim = bound(c, q, tk, tv, parent, n_nodes, ref, lens_lists, (out_dtype or f32) == bf16, kw.get("scale"))
    got = out.float().cpu().numpy().astype(np.float64)
    if n_nodes is not None:                       # rows of nodes that do not exist are left alone
        for bb, m in enumerate(n_nodes):
            assert (got[:, bb, :, m:] == -7.0).all()
    assert np.isfinite(got).all() and (np.abs(got - ref) <= lim).all(), np.max(np.abs(got - ref) / lim)


TREE_CASES = [
    # dtype, d, Hq, Hkv, L, lens, N, tree, nodes per tree
    (f32, 64, 4, 4, 1, [70, 0, 31, 32], 5, "tree", None),
    (f32, 128, 6, 2, 2, [33, 1], 17, "tree", [17, 9]),
    (f32, 64, 4, 1, 1, [100], 33, "chain", None),
    (f32, 128, 2, 1, 1, [700, 300], 1, "chain", None),
    (f32, 64, 28, 4, 1, [64, 5], 128, "tree", [128, 0]),
    (bf16, 128, 12, 2, 2, [300, 64, 0, 63], 16, "tree", [16, 1, 7, 0]),
    (bf16, 128, 12, 2, 1, [65, 129], 1, "chain", None),
    (bf16, 128, 28, 4, 1, [200, 17], 33, "tree", None),
    (bf16, 128, 12, 2, 1, [257], 64, "tree", None),
    (bf16, 128, 4, 4, 2, [90, 128], 128, "chain", [128, 65]),
    (bf16, 128, 16, 1, 1, [64], 20, "star", None),
    (bf16, 128, 40, 2, 1, [1, 190], 8, "tree", None),
    (bf16, 64, 8, 2, 2, [130, 7], 12, "tree", [12, 3]),
    (bf16, 64, 4, 4, 1, [0, 64, 65], 70, "tree", None),
]


@pytest.mark.parametrize("i", range(len(TREE_CASES)))
def test_tree_attn_matches_oracle(i):
    dtype, d, Hq, Hkv, L, lens, N, kind, nodes = TREE_CASES[i]
    c, q, tk, tv, parent, n_nodes = case(dtype, d, Hq, Hkv, L, lens, N, kind, seed=10 * i, n_nodes=nodes)
    check_tree(c, q, tk, tv, parent, n_nodes)
    if dtype == bf16:
        check_tree(c, q, tk, tv, parent, n_nodes, out_dtype=bf16)


# launches: 1 where a cluster of CTAs shares a unit, 2 where units are cut and joined by a second kernel
@pytest.mark.parametrize("dtype,d,Hq,Hkv,N,T,launches", [(bf16, 128, 12, 2, 16, 5000, 1), (bf16, 128, 12, 2, 64, 3001, 1), (bf16, 128, 2, 2, 1, 9000, 1),
                                                         (bf16, 64, 4, 1, 9, 4096, 1), (f32, 128, 4, 2, 7, 2500, 2), (f32, 64, 2, 2, 40, 1500, 2),
                                                         (bf16, 128, 12, 2, 16, 9001, 1), (bf16, 128, 12, 2, 64, 12000, 2), (bf16, 64, 4, 1, 9, 10000, 1),
                                                         (bf16, 128, 12, 2, 16, 16001, 2), (bf16, 64, 4, 1, 9, 20000, 2), (bf16, 128, 2, 2, 1, 16100, 2)])
def test_tree_attn_splits_a_long_cache(dtype, d, Hq, Hkv, N, T, launches):
    c, q, tk, tv, parent, n_nodes = case(dtype, d, Hq, Hkv, 1, [T, T // 3], N, "tree", seed=T, n_nodes=[N, max(1, N // 2)])
    b = ngc()
    dc = b.NgcCache(c.k.cuda(), c.v.cuda(), c.seq_off.cuda(), c.lens.cuda(), Hq, T)
    assert b.tree_attn_launches(dc, N) == launches
    check_tree(c, q, tk, tv, parent, n_nodes)


@pytest.mark.parametrize("d,L,B,Hq,Hkv,N,T,launches", [(128, 2, 330, 2, 2, 3, 150, 1), (64, 1, 700, 2, 2, 2, 70, 1), (128, 1, 80, 2, 2, 65, 300, 2),
                                                       (128, 1, 310, 130, 1, 2, 40, 1), (128, 3, 90, 2, 1, 1, 700, 2), (128, 1, 60, 8, 4, 90, 130, 2)])
def test_tree_attn_deals_out_many_units(d, L, B, Hq, Hkv, N, T, launches):
    """More (layer, sequence, KV head, row block) units than SMs: whole units dealt out (one launch), or units cut where the
    deal falls and joined (two); ragged lengths with empty caches, full ones and empty trees among them."""
    rng = np.random.default_rng(B)
    lens = rng.integers(0, T + 1, B)
    lens[:4] = [0, T, 0, T]
    nodes = rng.integers(0, N + 1, B)
    nodes[:4] = [N, N, 0, 0]
    c, q, tk, tv, parent, n_nodes = case(bf16, d, Hq, Hkv, L, lens.tolist(), N, "tree", seed=B, capacity=T, n_nodes=nodes)
    b = ngc()
    dc = b.NgcCache(c.k.cuda(), c.v.cuda(), c.seq_off.cuda(), c.lens.cuda(), Hq, T)
    assert b.tree_attn_launches(dc, N) == launches
    check_tree(c, q, tk, tv, parent, n_nodes)


@pytest.mark.parametrize("dtype,d", [(f32, 64), (bf16, 128), (bf16, 64)])
def test_tree_attn_takes_nothing_from_dead_rows_and_other_branches(dtype, d):
    """Cache rows beyond the length, nodes beyond the tree and (for the rows that do not see them) nodes of other
    branches hold infinities and NaN: no finite row may change, and a row that sees such a node shows it."""
    L, Hq, Hkv, N, lens = 1, 4, 2, 70, [100, 64]
    c, q, tk, tv, parent, n_nodes = case(dtype, d, Hq, Hkv, L, lens, N, "tree", seed=3, capacity=192, n_nodes=[70, 66])
    clean, st = run_tree(c, q, tk, tv, parent, n_nodes)
    c2 = c.clone()
    so = c.seq_off
    for b, n in enumerate(lens):
        c2.k[:, :, so[b] + n:so[b + 1]] = float("nan")
        c2.v[:, :, so[b] + n:so[b + 1]] = float("inf")
    tk2, tv2 = tk.clone(), tv.clone()
    tk2[:, 1, :, 66:] = float("nan")
    tv2[:, 1, :, 66:] = float("-inf")
    same, st2 = run_tree(c2, q, tk2, tv2, parent, n_nodes)
    assert st == 0 and st2 == 0 and torch.equal(clean, same)
    bad = {5: float("inf"), 40: float("nan"), 69: float("-inf")}       # a node of each kind, in the tree's first and second tile
    for i, x in bad.items():
        tv2[:, 0, :, i, 1] = x
    out, st3 = run_tree(c2, q, tk2, tv2, parent, n_nodes)
    hit = np.array([[i in draft.ancestors(parent[0], j) for i in bad] for j in range(N)]).any(-1)
    assert st3 == 0 and hit.sum() >= 3 and (~hit).sum() >= 3
    got, ref = out[:, 0].cpu().numpy(), clean[:, 0].cpu().numpy()
    assert np.array_equal(got[:, :, ~hit], ref[:, :, ~hit])
    assert not np.isfinite(got[:, :, hit, 1]).any()
    keep = [ch for ch in range(d) if ch != 1]
    assert np.array_equal(got[:, :, hit][..., keep], ref[:, :, hit][..., keep])
    # a key of infinities: only rows that see node 5 may notice
    tk3 = tk.clone()
    tk3[:, 0, :, 5] = float("inf")
    out, _ = run_tree(c, q, tk3, tv, parent, n_nodes)
    sees5 = np.array([5 in draft.ancestors(parent[0], j) for j in range(N)])
    assert np.array_equal(out[:, 0].cpu().numpy()[:, :, ~sees5], ref[:, :, ~sees5])


@pytest.mark.parametrize("dtype,d", [(f32, 64), (bf16, 128)])
def test_tree_attn_shows_a_nan_that_a_row_sees(dtype, d):
    c, q, tk, tv, parent, n_nodes = case(dtype, d, 4, 2, 1, [70], 3, "star", seed=8)
    c.k[0, 0, 5, 0] = float("nan")
    out, st = run_tree(c, q, tk, tv, parent, n_nodes)
    assert st == 0 and torch.isnan(out[:, :, :2]).all() and torch.isfinite(out[:, :, 2:]).all()


@pytest.mark.parametrize("dtype,d,N", [(f32, 64, 6), (bf16, 128, 6), (bf16, 128, 40)])
def test_tree_attn_layer_ranges_scale_and_lengths_per_list(dtype, d, N):
    L, Hq, Hkv, lens = 3, 6, 2, [150, 40]
    c, q, tk, tv, parent, n_nodes = case(dtype, d, Hq, Hkv, L, lens, N, "tree", seed=5, capacity=200)
    check_tree(c, q, tk, tv, parent, n_nodes, scale=0.03)
    whole, _ = run_tree(c, q, tk, tv, parent, n_nodes)
    part, st = run_tree(c, q, tk, tv, parent, n_nodes, layer_begin=1, layer_end=2)
    assert st == 0 and (part[0] == -7).all() and (part[2] == -7).all()
    lim = torch.as_tensor(bound(c, q, tk, tv, parent, n_nodes, whole.cpu().numpy())[1]).cuda() * 2     # each off by its own bound
    assert (torch.abs(part[1].double() - whole[1].double()) <= lim).all()
    rng = np.random.default_rng(1)
    for lists in (1, 2):
        G = oracle.lists_G(lists, L, Hkv)
        c.lens = torch.as_tensor(rng.integers(0, 201, (2, G)).astype(np.int32))
        check_tree(c, q, tk, tv, parent, n_nodes, lens_lists=lists)


@pytest.mark.parametrize("T", [64, 4000, 16000])   # one part, a cluster, several parts
@pytest.mark.parametrize("dtype,d", [(f32, 64), (bf16, 128)])
def test_tree_attn_skips_refused_sequences(dtype, d, T):
    N = 9
    c, q, tk, tv, parent, _ = case(dtype, d, 4, 2, 1, [T, T, T, T], N, "tree", seed=4)
    good, st = run_tree(c, q, tk, tv, parent, None)
    assert st == 0
    # A long bf16 cache is cut into parts at places that depend on all the sequences' lengths, so the same row may come
    # out of another grouping of the same sums: each of the two is within its bound of the exact value, hence they
    # are within twice that of one another.  Everything else is the same to the bit.
    ref = draft.tree_attn(synth.to_numpy(c.k), synth.to_numpy(c.v), c.seq_off.numpy(), c.lens.numpy(), synth.to_numpy(q), synth.to_numpy(tk),
                          synth.to_numpy(tv), parent)
    lim = torch.as_tensor(2 * bound(c, q, tk, tv, parent, None, ref)).cuda() * int(dtype == bf16 and T > 64)

    def same(out, seqs):
        return bool((torch.abs(out[:, seqs].double() - good[:, seqs].double()) <= lim[:, seqs]).all())
    for where, val in (((1, 0), 0), ((1, 4), 4), ((1, 4), 7), ((1, 8), -1), ((1, 3), -2)):
        p2 = parent.copy()
        p2[where] = val
        out, st = run_tree(c, q, tk, tv, p2, None)
        assert st == 8 and (out[:, 1] == -7).all() and same(out, [0, 2, 3])
    out, st = run_tree(c, q, tk, tv, parent, np.array([N, -1, N + 1, N], np.int32))
    assert st == 8 and (out[:, 1:3] == -7).all() and same(out, [0, 3])
    lens = c.lens.clone()
    lens[0], lens[2] = -1, T + 1
    out, st = run_tree(c, q, tk, tv, parent, None, lens=lens)
    assert st == 1 and (out[:, [0, 2]] == -7).all() and same(out, [1, 3])


def to_pages(c, page, lists, seed, per_list):
    """The contiguous host cache behind random page tables; free pages hold junk."""
    b = ngc()
    L, Hkv, R, d = c.k.shape
    B, G = len(c.seq_off) - 1, oracle.lists_G(lists, L, Hkv)
    so = c.seq_off.numpy()
    cap = int(so[1] - so[0])
    pages = cap // page
    rng = np.random.default_rng(seed)
    table = np.stack([[rng.permutation(pages) for _ in range(G)] for _ in range(B)]).astype(np.int32)
    kp = torch.full((L, Hkv, B * pages, page, d), float("nan"), dtype=c.k.dtype)
    vp = kp.clone()
    lens = c.lens.numpy()
    for bb in range(B):
        for l in range(L):
            for h in range(Hkv):
                gi = (0, l, l * Hkv + h)[lists]
                n = int(lens[bb, gi] if per_list else lens[bb])
                for t in range(min(n, cap)):
                    r = (bb * pages + table[bb, gi, t // page], t % page)
                    kp[l, h][r], vp[l, h][r] = c.k[l, h, so[bb] + t], c.v[l, h, so[bb] + t]
    return b.NgcPagedCache(kp.cuda(), vp.cuda(), torch.as_tensor(table).cuda(), c.lens.clone().cuda(), c.Hq, lists)


def from_pages(pc, page, lists, lens, so, L, Hkv):
    """Host arrays [L][Hkv][R][d] of the alive rows (zeros elsewhere), with R = seq_off[-1]."""
    k, v, table = pc.k.cpu(), pc.v.cpu(), pc.page_table.cpu().numpy()
    pages, d = table.shape[2], k.shape[-1]
    out = [torch.zeros((L, Hkv, int(so[-1]), d), dtype=k.dtype) for _ in range(2)]
    for bb in range(table.shape[0]):
        for l in range(L):
            for h in range(Hkv):
                gi = (0, l, l * Hkv + h)[lists]
                n = int(lens[bb, gi] if lens.ndim == 2 else lens[bb])
                for t in range(n):
                    for o, a in zip(out, (k, v)):
                        o[l, h, so[bb] + t] = a[l, h, bb * pages + table[bb, gi, t // page], t % page]
    return [synth.to_numpy(o) for o in out]


PAGED = [(32, 0, False, 12, 2, 16, [70, 0, 128]), (32, 1, True, 28, 4, 33, [96, 31]), (64, 2, True, 4, 2, 70, [64, 65]),
         (64, 0, False, 2, 2, 1, [190, 1]), (32, 1, False, 16, 2, 5, [33, 191])]


@pytest.mark.parametrize("page,lists,per_list,Hq,Hkv,N,lens", PAGED)
def test_paged_tree_attn_matches_oracle(page, lists, per_list, Hq, Hkv, N, lens):
    b = ngc()
    L, d = 2, 128
    c, q, tk, tv, parent, _ = case(bf16, d, Hq, Hkv, L, lens, N, "tree", seed=page + N, capacity=192)
    if per_list:
        rng = np.random.default_rng(N)
        c.lens = torch.as_tensor(rng.integers(0, 193, (len(lens), oracle.lists_G(lists, L, Hkv))).astype(np.int32))
    pc = to_pages(c, page, lists, 7, per_list)
    ll = lists if per_list else 0
    ref = draft.tree_attn(synth.to_numpy(c.k), synth.to_numpy(c.v), c.seq_off.numpy(), c.lens.numpy(), synth.to_numpy(q), synth.to_numpy(tk),
                          synth.to_numpy(tv), parent, lens_lists=ll)
    out = torch.full(q.shape, -7.0, dtype=f32, device="cuda")
    ws = b.alloc_workspace(b.workspace_bytes(b.OP_TREE_ATTN, pc.as_contiguous_desc(), n_max=N))
    st = b.new_status()
    b.ngc_tree_attn_paged(pc, q.cuda(), tk.cuda(), tv.cuda(), torch.as_tensor(parent).cuda(), out, ws=ws, status=st)
    torch.cuda.synchronize()
    assert status_value(st) == 0
    lim = bound(c, q, tk, tv, parent, None, ref, ll)
    got = out.cpu().numpy().astype(np.float64)
    assert (np.abs(got - ref) <= lim).all(), np.max(np.abs(got - ref) / lim)


def test_paged_bad_page_entry_is_reported_and_stays_with_its_sequence():
    b = ngc()
    c, q, tk, tv, parent, _ = case(bf16, 128, 4, 2, 1, [100, 100], 4, "tree", seed=1, capacity=128)
    dev = [x.cuda() for x in (q, tk, tv, torch.as_tensor(parent))]
    outs = []
    for entry in (None, -1, 2, 1 << 30):
        pc = to_pages(c, 64, 0, 7, False)
        if entry is not None:
            pc.page_table[1, 0, 1] = entry
        out = torch.zeros(q.shape, dtype=f32, device="cuda")
        st = b.new_status()
        ws = b.alloc_workspace(b.workspace_bytes(b.OP_TREE_ATTN, pc.as_contiguous_desc(), n_max=4))
        b.ngc_tree_attn_paged(pc, *dev, out, ws=ws, status=st)
        torch.cuda.synchronize()
        assert status_value(st) == (0 if entry is None else 11)
        outs.append(out)
        if entry is not None:
            assert torch.equal(out[:, 0], outs[0][:, 0])
            # commit and fork leave the sequence with the bad page as it was
            before = [x.clone() for x in (pc.k, pc.v, pc.lens)]
            path = torch.tensor([[0, 1, -1, -1]] * 2, dtype=torch.int32).cuda()
            st.zero_()
            b.ngc_commit_draft_paged(pc, dev[1], dev[2], path, torch.tensor([0, 2], dtype=torch.int32).cuda(), status=st)
            assert status_value(st) == 11
            st.zero_()
            b.ngc_fork_pages(pc, torch.tensor([1, -1], dtype=torch.int32).cuda(), status=st)
            assert status_value(st) == 11
            st.zero_()
            b.ngc_fork_pages(pc, torch.tensor([-1, 0], dtype=torch.int32).cuda(), status=st)
            assert status_value(st) == 11
            for x, y in zip(before, (pc.k, pc.v, pc.lens)):
                assert torch.equal(x.view(torch.int16) if x.dtype == bf16 else x, y.view(torch.int16) if y.dtype == bf16 else y)


def test_tree_attn_offsets_beyond_32_bits():
    """Two planes of 9 million rows: element offsets pass 2^31 in the second one, and its last rows are the ones read."""
    b = ngc()
    Hq, Hkv, d, N, T, cap = 4, 2, 128, 5, 150, 9_000_000
    small, q, tk, tv, parent, _ = case(bf16, d, Hq, Hkv, 1, [T], N, "tree", seed=2)
    k = torch.empty((1, Hkv, cap, d), dtype=bf16, device="cuda")
    v = torch.empty_like(k)
    k[:, :, cap - 1000:], v[:, :, cap - 1000:] = float("nan"), float("nan")
    k[:, :, cap - 1000:cap - 1000 + T], v[:, :, cap - 1000:cap - 1000 + T] = small.k.cuda(), small.v.cuda()
    so = torch.tensor([0, cap - 1000, cap])
    pad = [torch.cat([x, x], 1) for x in (q, tk, tv)]
    cache = b.NgcCache(k, v, so.cuda(), torch.tensor([0, T], dtype=torch.int32).cuda(), Hq, 1000)
    out = torch.zeros(pad[0].shape, dtype=f32, device="cuda")
    st = b.new_status()
    ws = b.alloc_workspace(b.workspace_bytes(b.OP_TREE_ATTN, cache, n_max=N))
    b.ngc_tree_attn(cache, *[x.cuda() for x in pad], torch.as_tensor(np.concatenate([parent, parent])).cuda(), out, ws=ws, status=st)
    ref = draft.tree_attn(synth.to_numpy(small.k), synth.to_numpy(small.v), np.array([0, T]), np.array([T]), synth.to_numpy(q),
                          synth.to_numpy(tk), synth.to_numpy(tv), parent)
    lim = bound(small, q, tk, tv, parent, None, ref)
    assert (np.abs(out[:, 1].cpu().numpy() - ref[:, 0]) <= lim[:, 0]).all()
    # the append and a fork at the same place
    path = torch.tensor([[-1] * N, [0, 2, 4, -1, -1]], dtype=torch.int32).cuda()
    b.ngc_commit_draft(cache, pad[1].cuda(), pad[2].cuda(), path, torch.tensor([0, 3], dtype=torch.int32).cuda(), status=st)
    assert torch.equal(k[:, :, cap - 1000 + T:cap - 1000 + T + 3], tk[:, 0, :, [0, 2, 4]].cuda())
    b.ngc_fork_kv(cache, torch.tensor([1, -1], dtype=torch.int32).cuda(), status=st)
    assert status_value(st) == 0 and cache.lens.tolist() == [T + 3, T + 3]
    assert torch.equal(k[:, :, :T + 3], k[:, :, cap - 1000:cap - 1000 + T + 3]) and torch.equal(v[:, :, :T + 3], v[:, :, cap - 1000:cap - 1000 + T + 3])


# ---------------------------------------------------------------- verification

def run_verify(tokens, parent, target, u, dr=None, n_nodes=None, greedy=0):
    b = ngc()
    B, N, V = target.shape

    def dev(a, t):
        return None if a is None else torch.as_tensor(np.ascontiguousarray(a, t)).cuda()
    path = torch.full((B, N), 99, dtype=torch.int32, device="cuda")
    n_path, nxt = (torch.full((B,), 99, dtype=torch.int32, device="cuda") for _ in range(2))
    st = b.new_status()
    b.ngc_verify_draft(dev(tokens, np.int32), dev(parent, np.int32), dev(target, np.float32), dev(u, np.float32), path, n_path, nxt,
                       dev(dr, np.float32), dev(n_nodes, np.int32), greedy, status=st)
    return path.cpu().numpy(), n_path.cpu().numpy(), nxt.cpu().numpy(), status_value(st)


def draft_case(B, N, V, kind, mode, seed, std=2.0, noise=0.6):
    rng = np.random.default_rng(seed)
    z = rng.standard_normal((B, N, V)) * std

    def soft(x):
        e = np.exp(x - x.max(-1, keepdims=True))
        return (e / e.sum(-1, keepdims=True)).astype(np.float32)
    p, q = soft(z), soft(z + noise * rng.standard_normal((B, N, V)))
    parent = trees(B, N, kind, seed)
    tokens = np.zeros((B, N), np.int32)
    for b in range(B):
        seen = {}
        for i in range(1, N):
            a = parent[b, i]
            if mode == "draft":
                cdf = np.cumsum(q[b, a].astype(np.float64))
                tokens[b, i] = min(V - 1, np.searchsorted(cdf, rng.random() * cdf[-1], side="right"))
            else:
                r = seen[a] = seen.get(a, -1) + 1
                tokens[b, i] = np.argsort(-q[b, a], kind="stable")[min(r, V - 1)]
    return tokens, parent, p, q if mode == "draft" else None, rng.random((B, N)).astype(np.float32)


def check_verify(tokens, parent, p, q, u, n_nodes=None, greedy=0):
    ref = draft.verify_draft(tokens, parent, p, u, q, n_nodes, greedy)
    got = run_verify(tokens, parent, p, u, q, n_nodes, greedy)
    assert np.array_equal(got[0], ref[0]) and np.array_equal(got[1], ref[1]) and np.array_equal(got[2], ref[2])
    assert (got[3] == 0) == (not ref[3].any()) and (got[3] == 0 or got[3] in ref[3])
    return ref


@pytest.mark.parametrize("mode", ["draft", "point", "greedy"])
@pytest.mark.parametrize("B,N,V,kind", [(1, 1, 1, "chain"), (3, 4, 2, "star"), (7, 5, 33, "chain"), (40, 17, 1000, "tree"), (5, 128, 257, "star"),
                                        (3, 9, 50001, "tree"), (2, 6, 131072, "chain"), (4, 128, 999, "tree")])
def test_verify_matches_oracle(B, N, V, kind, mode):
    tokens, parent, p, q, u = draft_case(B, N, V, kind, mode, seed=B * 1000 + N)
    rng = np.random.default_rng(1)
    ref = check_verify(tokens, parent, p, q, u, greedy=int(mode == "greedy"))
    check_verify(tokens, parent, p, q, u, n_nodes=rng.integers(0, N + 1, B), greedy=int(mode == "greedy"))
    if N > 1 and B > 5:
        assert ref[1].max() > 1


def test_verify_edges():
    tokens, parent, p, q, u = draft_case(6, 4, 300, "star", "draft", 3)
    for val in (0.0, 1.0 - 2.0 ** -24):
        check_verify(tokens, parent, p, q, np.full_like(u, val))
        check_verify(tokens, parent, p, None, np.full_like(u, val))
    check_verify(tokens, parent, p, p, u)                                   # the draft is the target: everything is accepted
    check_verify(tokens, parent, p, p, np.full_like(u, 1.0 - 2.0 ** -24))
    z = np.zeros_like(p)
    z[..., 7] = 1.0                                                         # all mass on one token
    check_verify(tokens, parent, z, q, u)
    check_verify(np.full_like(tokens, 7), parent, z, None, u)
    check_verify(np.full_like(tokens, 9), parent, z, z, u)                  # a child the draft itself could not have drawn
    tie = np.round(p * 50) / 50                                             # many equal maxima: the lowest index counts
    check_verify(tokens, parent, tie, None, u, greedy=1)
    check_verify(np.full_like(tokens, 5), parent, np.full_like(p, -np.inf), None, u, greedy=1)
    same = np.broadcast_to(tokens[:, 1:2], tokens.shape)                    # the same token under every child
    check_verify(same, parent, p, q, u)
    check_verify(same, parent, p, None, np.full_like(u, 0.999))


def test_verify_reports_what_it_cannot_use():
    tokens, parent, p, q, u = draft_case(3, 5, 64, "tree", "draft", 4)
    u[:] = 0.999999
    good = draft.verify_draft(tokens, parent, p, u, q)
    def expect(status, t=tokens, pa=parent, pp=p, qq=q, uu=u, n=None, greedy=0):
        got = run_verify(t, pa, pp, uu, qq, n, greedy)
        assert got[3] == status and (got[0][1] == -1).all() and got[1][1] == 0 and got[2][1] == -1
        if not greedy:
            for g, r in zip(got[:3], good[:3]):
                assert np.array_equal(g[[0, 2]], r[[0, 2]])
    for x in (-1, 64, 1 << 30):
        t = tokens.copy()
        t[1, 3] = x
        expect(8, t=t)
    for at, x in ((0, 0), (2, 2), (3, -1), (4, 9)):
        pa = parent.copy()
        pa[1, at] = x
        expect(8, pa=pa)
    expect(8, n=np.array([5, 6, 5]))
    for x in (0.0, np.nan, np.inf):
        pp = p.copy()
        pp[1] = x
        expect(9, pp=pp)
    qq = q.copy()
    qq[1] = np.nan
    expect(9, qq=qq)
    pp = p.copy()
    pp[1, 0, 60] = np.nan
    expect(9, pp=pp, qq=None, greedy=1)
    # an empty tree is no error
    got = run_verify(tokens, parent, p, u, q, np.array([5, 0, 5]))
    assert got[3] == 0 and got[1][1] == 0 and got[2][1] == -1 and (got[0][1] == -1).all()


# ---------------------------------------------------------------- commit and fork

def device_cache(c, lens_lists=0):
    b = ngc()
    cap = int((c.seq_off[1:] - c.seq_off[:-1]).max())
    return b.NgcCache(c.k.cuda(), c.v.cuda(), c.seq_off.cuda(), c.lens.cuda(), c.Hq, cap, lens_lists)


@pytest.mark.parametrize("dtype,d,L,Hkv,N,cap,lens_lists", [(bf16, 128, 2, 2, 8, [40, 64, 33], 0), (f32, 64, 1, 3, 1, [5, 9, 4], 0),
                                                            (bf16, 64, 3, 2, 128, [300, 200, 130], 1), (f32, 128, 2, 2, 5, [50, 60, 70], 2),
                                                            (bf16, 128, 28, 2, 16, [64, 64, 64], 1)])
def test_commit_matches_oracle_bit_for_bit(dtype, d, L, Hkv, N, cap, lens_lists):
    b = ngc()
    B, rng = 3, np.random.default_rng(N)
    c = synth.make_cache(L, B, Hkv, Hkv, d, dtype, [0] * B, capacity=cap, seed=N)
    room = np.array([x - N for x in cap])
    shape = (B,) if not lens_lists else (B, oracle.lists_G(lens_lists, L, Hkv))
    c.lens = torch.as_tensor((rng.random(shape) * (room + 1).reshape((-1,) + (1,) * (len(shape) - 1))).astype(np.int32))
    tk, tv = (synth.normal((L, B, Hkv, N, d), s, dtype) for s in (3, 4))
    n_path = np.array([N, rng.integers(0, N + 1), 0], np.int32)
    path = np.full((B, N), -1, np.int32)
    for bb in range(B):
        path[bb, :n_path[bb]] = np.sort(rng.choice(N, n_path[bb], replace=False))
    dc = device_cache(c, lens_lists)
    st = b.new_status()
    for _ in range(2):                     # the second append starts where the first ended, or is refused as a whole
        k, v, ln = synth.to_numpy(dc.k), synth.to_numpy(dc.v), dc.lens.cpu().numpy()
        rk, rv, rl, rs = draft.commit_draft(k, v, c.seq_off.numpy(), ln, synth.to_numpy(tk), synth.to_numpy(tv), path, n_path, lens_lists)
        st.zero_()
        b.ngc_commit_draft(dc, tk.cuda(), tv.cuda(), torch.as_tensor(path).cuda(), torch.as_tensor(n_path).cuda(), status=st)
        assert (status_value(st) == 0) == (not rs.any()) and (status_value(st) == 0 or status_value(st) in rs)
        assert np.array_equal(synth.to_numpy(dc.k), rk) and np.array_equal(synth.to_numpy(dc.v), rv)
        assert np.array_equal(dc.lens.cpu().numpy(), rl)


def test_commit_refuses_bad_paths_and_full_strips_whole():
    b = ngc()
    L, B, Hkv, d, N = 2, 4, 2, 64, 6
    for lens_lists in (0, 1):
        c = synth.make_cache(L, B, Hkv, Hkv, d, f32, [10] * B, capacity=16, seed=1)
        if lens_lists:
            c.lens = torch.tensor([[10, 3], [10, 3], [10, 15], [10, 3]], dtype=torch.int32)
        else:
            c.lens = torch.tensor([10, 10, 15, 10], dtype=torch.int32)
        tk, tv = (synth.normal((L, B, Hkv, N, d), s, f32) for s in (3, 4))
        for bad in ([2, 2, -1, -1, -1, -1], [3, 1, -1, -1, -1, -1], [0, 6, -1, -1, -1, -1], [-1, 2, -1, -1, -1, -1], None):
            path = np.array([[0, 2, 4, -1, -1, -1]] * B, np.int32)
            n_path = np.array([3, 2, 2, 1], np.int32)
            if bad is None:
                n_path[1] = N + 1
            else:
                path[1] = bad
            dc = device_cache(c, lens_lists)
            st = b.new_status()
            b.ngc_commit_draft(dc, tk.cuda(), tv.cuda(), torch.as_tensor(path).cuda(), torch.as_tensor(n_path).cuda(), status=st)
            rk, rv, rl, rs = draft.commit_draft(c.k.numpy(), c.v.numpy(), c.seq_off.numpy(), c.lens.numpy(), tk.numpy(), tv.numpy(), path, n_path, lens_lists)
            assert rs.tolist() == [0, 8, 4, 0] and status_value(st) in (4, 8)
            assert np.array_equal(dc.k.cpu().numpy(), rk) and np.array_equal(dc.v.cpu().numpy(), rv) and np.array_equal(dc.lens.cpu().numpy(), rl)


@pytest.mark.parametrize("page,lists,per_list", [(32, 0, False), (32, 1, True), (64, 2, True), (64, 1, False)])
def test_paged_commit_and_fork_match_oracle(page, lists, per_list):
    b = ngc()
    L, Hkv, d, N, B = 2, 2, 128, 9, 4
    c = synth.make_cache(L, B, Hkv, Hkv, d, bf16, [0] * B, capacity=192, seed=page)
    rng = np.random.default_rng(page + lists)
    shape = (B, oracle.lists_G(lists, L, Hkv)) if per_list else (B,)
    c.lens = torch.as_tensor(rng.integers(0, 180, shape).astype(np.int32))
    c.lens[2] = 190                                                        # full after two more rows
    tk, tv = (synth.normal((L, B, Hkv, N, d), s, bf16) for s in (3, 4))
    pc = to_pages(c, page, lists, 3, per_list)
    ll, so = lists if per_list else 0, c.seq_off.numpy()
    path = np.full((B, N), -1, np.int32)
    path[0, :5], path[1, :9], path[2, :3] = [0, 1, 3, 6, 8], range(9), [0, 1, 2]
    n_path = np.array([5, 9, 3, 0], np.int32)
    k, v, ln, rs = draft.commit_draft(synth.to_numpy(c.k), synth.to_numpy(c.v), so, c.lens.numpy(), synth.to_numpy(tk), synth.to_numpy(tv), path, n_path, ll)
    assert rs.tolist() == [0, 0, 4, 0]
    st = b.new_status()
    b.ngc_commit_draft_paged(pc, tk.cuda(), tv.cuda(), torch.as_tensor(path).cuda(), torch.as_tensor(n_path).cuda(), status=st)
    assert status_value(st) == 4

    def same(k, v, ln):
        assert np.array_equal(pc.lens.cpu().numpy(), ln)
        got = from_pages(pc, page, lists, ln, so, L, Hkv)
        for a, r in zip(got, (k, v)):
            for bb in range(B):
                for l in range(L):
                    for h in range(Hkv):
                        n = draft.strip_len(ln, ll, bb, l, h, Hkv)
                        assert np.array_equal(a[l, h, so[bb]:so[bb] + n], r[l, h, so[bb]:so[bb] + n])
    same(k, v, ln)
    src = np.array([-1, 0, 2, 0], np.int32)
    k, v, ln, rs = draft.fork(k, v, so, ln, src, ll)
    assert not rs.any()
    st.zero_()
    table = pc.page_table.clone()
    b.ngc_fork_pages(pc, torch.as_tensor(src).cuda(), status=st)
    assert status_value(st) == 0 and torch.equal(table, pc.page_table)
    same(k, v, ln)


@pytest.mark.parametrize("dtype,d,lens_lists", [(bf16, 128, 0), (f32, 64, 1), (bf16, 64, 2), (f32, 128, 0)])
def test_fork_matches_oracle_bit_for_bit(dtype, d, lens_lists):
    b = ngc()
    L, Hkv, cap = 2, 2, [130, 130, 20, 130, 200, 131, 1, 300, 140, 140]
    B = len(cap)
    c = synth.make_cache(L, B, Hkv, Hkv, d, dtype, [1] * B, capacity=cap, seed=d)
    rng = np.random.default_rng(d)
    shape = (B,) if not lens_lists else (B, oracle.lists_G(lens_lists, L, Hkv))
    lens = np.minimum(rng.integers(0, 131, shape), np.array(cap).reshape((-1,) + (1,) * (len(shape) - 1))).astype(np.int32)
    lens[0], lens[7] = 129, 250
    lens[8], lens[6] = 0, -3                         # an empty source; a source with a length that is none
    c.lens = torch.as_tensor(lens)
    src = np.array([-1, 0, 0, 7, 7, 0, -1, -1, -1, 8], np.int32)      # 2 is too small for 0, 3 for 7
    for s in (src, np.where(np.arange(B) == 9, 6, src), np.where(np.arange(B) == 9, 4, src), np.where(np.arange(B) == 5, B, src),
              np.where(np.arange(B) == 5, -2, src), np.arange(B)):
        s = s.astype(np.int32)
        dc = device_cache(c, lens_lists)
        st = b.new_status()
        b.ngc_fork_kv(dc, torch.as_tensor(s).cuda(), status=st)
        rk, rv, rl, rs = draft.fork(synth.to_numpy(c.k), synth.to_numpy(c.v), c.seq_off.numpy(), lens, s, lens_lists)
        assert (status_value(st) == 0) == (not rs.any()) and (status_value(st) == 0 or status_value(st) in rs)
        assert np.array_equal(synth.to_numpy(dc.k), rk) and np.array_equal(synth.to_numpy(dc.v), rv) and np.array_equal(dc.lens.cpu().numpy(), rl)


# ---------------------------------------------------------------- together

@pytest.mark.parametrize("dtype,d,Hq,Hkv", [(bf16, 128, 12, 2), (f32, 64, 4, 4)])
def test_forked_rollouts_advance_by_drafts_across_an_eviction(dtype, d, Hq, Hkv):
    """One prompt forked to its group, three draft steps (attention, verification, commit), an eviction round, two more
    draft steps: caches bit for bit and attention within its bound against the oracle all the way."""
    from paper_2604_18002_b200.rollout import NgcRollout
    L, B, N, V, T, K = 2, 4, 7, 501, 90, 60
    ro = NgcRollout(L, B, Hq, Hkv, d, dtype, 160, n_max=160, k_max=K, w=5)
    c = synth.make_cache(L, B, Hq, Hkv, d, dtype, [T, 0, 0, 0], capacity=160, seed=1)
    ro.cache.k.copy_(c.k)
    ro.cache.v.copy_(c.v)
    ro.cache.lens.copy_(c.lens)
    k, v, so, ln = synth.to_numpy(c.k), synth.to_numpy(c.v), c.seq_off.numpy(), c.lens.numpy().copy()
    src = np.array([-1, 0, 0, 0], np.int32)
    ro.fork(torch.as_tensor(src).cuda())
    k, v, ln, _ = draft.fork(k, v, so, ln, src)
    path = torch.empty((B, N), dtype=torch.int32, device="cuda")
    n_path, nxt = (torch.empty((B,), dtype=torch.int32, device="cuda") for _ in range(2))
    out = torch.empty((L, B, Hq, N, d), dtype=f32, device="cuda")
    advanced = 0
    for step in range(5):
        if step == 3:
            logits = synth.make_logits(B, 1, 160, seed=9)
            budget = np.full(B, K, np.int32)
            ro.eviction_round(torch.as_tensor(ln).cuda(), None, torch.as_tensor(budget).cuda(), 5, 0, logits=logits.cuda())
            _, ks, _, _ = oracle.sample_evict(logits.numpy(), ln, None, budget, K, 5, 0)
            k, v, ln, rc = oracle.compact_kv(k, v, so, ln, ks, budget, 0)
            assert rc == 0
        tokens, parent, p, q_d, u = draft_case(B, N, V, "tree", "draft", step, noise=0.3)
        q, tk, tv = (synth.normal((L, B, H, N, d), 100 + 7 * step + s, dtype) for H, s in ((Hq, 2), (Hkv, 3), (Hkv, 4)))
        dev = [torch.as_tensor(x).cuda() for x in (tokens, parent, p, u, q_d)]
        ro.draft_attention(q.cuda(), tk.cuda(), tv.cuda(), dev[1], out)
        ro.accept_draft(dev[0], dev[1], dev[2], dev[3], tk.cuda(), tv.cuda(), path, n_path, nxt, draft_probs=dev[4])
        ro.check_status()
        ref = draft.tree_attn(k, v, so, ln, synth.to_numpy(q), synth.to_numpy(tk), synth.to_numpy(tv), parent)
        host = synth.Cache(None, None, c.seq_off, torch.as_tensor(ln), L, B, Hq, Hkv, d)
        host.k, host.v = (torch.as_tensor(x.view(np.int16)).view(bf16) if dtype == bf16 else torch.as_tensor(x) for x in (k, v))
        assert (np.abs(out.cpu().numpy() - ref) <= bound(host, q, tk, tv, parent, None, ref)).all()
        r_path, r_n, r_next, _ = draft.verify_draft(tokens, parent, p, u, q_d)
        assert np.array_equal(path.cpu().numpy(), r_path) and np.array_equal(n_path.cpu().numpy(), r_n) and np.array_equal(nxt.cpu().numpy(), r_next)
        k, v, ln, _ = draft.commit_draft(k, v, so, ln, synth.to_numpy(tk), synth.to_numpy(tv), r_path, r_n)
        assert np.array_equal(ro.cache.lens.cpu().numpy(), ln)
        for b in range(B):
            s = slice(so[b], so[b] + ln[b])
            assert np.array_equal(synth.to_numpy(ro.cache.k)[:, :, s], k[:, :, s]) and np.array_equal(synth.to_numpy(ro.cache.v)[:, :, s], v[:, :, s])
        advanced += int(r_n.sum())
    assert advanced > 5 * B


def test_draft_step_in_a_graph_and_on_another_stream():
    """A captured step replays on new inputs; a call on a side stream gives what the same call on the main stream gives."""
    b = ngc()
    c, q, tk, tv, parent, _ = case(bf16, 128, 12, 2, 1, [2000, 700], 6, "tree", seed=1, capacity=2100)
    dc = device_cache(c)
    tokens, par, p, q_d, u = draft_case(2, 6, 300, "tree", "draft", 1)
    dq, dtk, dtv, dpar = q.cuda(), tk.cuda(), tv.cuda(), torch.as_tensor(parent).cuda()
    dtok, dp, dqd, du = (torch.as_tensor(x).cuda() for x in (tokens, p, q_d, u))
    out = torch.zeros(q.shape, dtype=f32, device="cuda")
    path = torch.empty((2, 6), dtype=torch.int32, device="cuda")
    n_path, nxt = (torch.empty((2,), dtype=torch.int32, device="cuda") for _ in range(2))
    ws = b.alloc_workspace(b.workspace_bytes(b.OP_TREE_ATTN, dc, n_max=6))
    st = b.new_status()

    def step():
        b.ngc_tree_attn(dc, dq, dtk, dtv, dpar, out, ws=ws, status=st)
        b.ngc_verify_draft(dtok, dpar, dp, du, path, n_path, nxt, dqd, status=st)
        b.ngc_commit_draft(dc, dtk, dtv, path, n_path, status=st)
    k0, v0, l0 = dc.k.clone(), dc.v.clone(), dc.lens.clone()

    def restore():
        dc.k.copy_(k0)
        dc.v.copy_(v0)
        dc.lens.copy_(l0)
    results = []
    for seed in (5, 6):
        dq.copy_(synth.normal(q.shape, seed, bf16))
        du.copy_(torch.as_tensor(np.random.default_rng(seed).random((2, 6)).astype(np.float32)))
        step()
        results.append([x.clone() for x in (out, path, n_path, nxt, dc.k, dc.lens)])
        restore()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    side = torch.cuda.Stream()
    for seed, want in zip((5, 6), results):
        dq.copy_(synth.normal(q.shape, seed, bf16))
        du.copy_(torch.as_tensor(np.random.default_rng(seed).random((2, 6)).astype(np.float32)))
        for x in (out, path, n_path, nxt):
            x.zero_()
        graph.replay()
        for x, w in zip((out, path, n_path, nxt, dc.k, dc.lens), want):
            assert torch.equal(x, w)
        restore()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            step()
        torch.cuda.current_stream().wait_stream(side)
        for x, w in zip((out, path, n_path, nxt, dc.k, dc.lens), want):
            assert torch.equal(x, w)
        restore()
    assert status_value(st) == 0


def test_rollout_refuses_to_allocate_while_capturing():
    """The first draft_attention with a node count allocates its workspace: inside a capture that is refused, and the capture
    of a call made before works."""
    from paper_2604_18002_b200.rollout import NgcRollout
    b = ngc()
    L, B, Hq, Hkv, d, N, T = 1, 2, 4, 2, 128, 4, 2000
    ro = NgcRollout(L, B, Hq, Hkv, d, bf16, T, n_max=T, k_max=8)
    ro.cache.k.normal_()
    ro.cache.v.normal_()
    ro.cache.lens.fill_(T)
    q, tk, tv = (torch.randn((L, B, H, N, d), device="cuda").to(bf16) for H in (Hq, Hkv, Hkv))
    parent = torch.as_tensor(trees(B, N, "tree", 1)).cuda()
    out = torch.empty((L, B, Hq, N, d), dtype=f32, device="cuda")
    q3, parent3 = q[:, :, :, :3].contiguous(), parent[:, :3].contiguous()
    ro.draft_attention(q, tk, tv, parent, out)
    ref = out.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ro.draft_attention(q, tk, tv, parent, out)
        with pytest.raises(b.NgcError, match="before capturing"):
            ro.draft_attention(q3, tk[:, :, :, :3].contiguous(), tv[:, :, :, :3].contiguous(), parent3, out[:, :, :, :3].contiguous())
    out.zero_()
    graph.replay()
    assert torch.equal(out, ref)
    ro.check_status()
