"""What the drafted-token calls must not touch, and rows at the edge of the number range.

(1) A spread of the calls' small parity cases on the bounds-checking build.  (2) Canaries: guard planes around K and V,
spare rows behind every sequence, guard elements behind outputs and workspaces.  (3) Two calls at once on two streams.
(4) Rows whose scores are NaN, all minus infinity, or huge."""
import numpy as np
import pytest
import torch

import test_gpu_draft as t_draft
from helpers import ngc, status_value
from oracle import draft
from paper_2604_18002_b200 import synth
from test_gpu_debug_build import PATTERN, assert_guards, debug_library, guarded, guarded_cache, planes_i16      # noqa: F401
from test_gpu_draft import bound, case, device_cache, draft_case, run_tree, trees

pytestmark = pytest.mark.gpu

bf16, f32 = torch.bfloat16, torch.float32

CASES = [(t_draft.test_tree_attn_matches_oracle, (i,)) for i in (0, 1, 4, 5, 7, 9, 12)] + [
    (t_draft.test_tree_attn_splits_a_long_cache, (bf16, 128, 12, 2, 64, 3001, 1)),
    (t_draft.test_tree_attn_splits_a_long_cache, (bf16, 128, 12, 2, 64, 12000, 2)),
    (t_draft.test_tree_attn_splits_a_long_cache, (f32, 64, 2, 2, 40, 1500, 2)),
    (t_draft.test_tree_attn_deals_out_many_units, (128, 2, 330, 2, 2, 3, 150, 1)),
    (t_draft.test_paged_tree_attn_matches_oracle, (32, 1, True, 28, 4, 33, [96, 31])),
    (t_draft.test_paged_bad_page_entry_is_reported_and_stays_with_its_sequence, ()),
    (t_draft.test_verify_matches_oracle, (5, 128, 257, "star", "draft")),
    (t_draft.test_commit_matches_oracle_bit_for_bit, (bf16, 64, 3, 2, 128, [300, 200, 130], 1)),
    (t_draft.test_paged_commit_and_fork_match_oracle, (32, 1, True)),
    (t_draft.test_fork_matches_oracle_bit_for_bit, (f32, 64, 1)),
]


@pytest.mark.parametrize("i", range(len(CASES)), ids=[f"{f.__name__}-{i}" for i, (f, _) in enumerate(CASES)])
def test_small_draft_case_on_the_bounds_checking_build(i, debug_library):      # noqa: F811
    fn, args = CASES[i]
    fn(*args)


# ------------------------------------------------------------------ canaries

def guarded_workspace(need, extra=4096):
    whole = torch.full((need + extra,), 0xAB, dtype=torch.uint8, device="cuda")
    return whole[:need], whole


@pytest.mark.parametrize("Hq,N,lens", [(12, 9, [700, 33, 257]), (12, 50, [300, 64, 1]), (2, 1, [5000, 2, 90]), (2, 3, [13000, 70, 1]), (2, 3, [20000, 70, 1])])
def test_canaries_survive_tree_attention_commit_and_fork(Hq, N, lens):
    b = ngc()
    L, B, Hkv, d = 2, 3, 2, 128
    cap = [max(lens) + N + 2] * B                              # 2 rows behind everything a sequence will hold
    host, dc, bufs, so = guarded_cache(L, B, Hq, Hkv, d, lens, cap, seed=41)
    q, tk, tv = (synth.normal((L, B, H, N, d), 50 + s, bf16) for H, s in ((Hq, 2), (Hkv, 3), (Hkv, 4)))
    parent, n_nodes = trees(B, N, "tree", 3), np.array([N, max(N - 4, 0), 1], np.int32)
    out, out_whole, out_fill = guarded((L, B, Hq, N, d), f32)
    ws, ws_whole = guarded_workspace(b.workspace_bytes(b.OP_TREE_ATTN, dc, n_max=N))
    st = b.new_status()
    k0, v0 = planes_i16(dc)
    dev = [x.cuda() for x in (q, tk, tv)]
    b.ngc_tree_attn(dc, *dev, torch.as_tensor(parent).cuda(), out, torch.as_tensor(n_nodes).cuda(), ws=ws, status=st)
    k1, v1 = planes_i16(dc)
    assert status_value(st) == 0 and np.array_equal(k0, k1) and np.array_equal(v0, v1) and dc.lens.tolist() == lens
    assert bool((out_whole[out.numel():] == out_fill).all()) and bool((ws_whole[ws.numel():] == 0xAB).all())
    ref = draft.tree_attn(synth.to_numpy(host.k), synth.to_numpy(host.v), so, host.lens.numpy(), *[synth.to_numpy(x) for x in (q, tk, tv)],
                          parent, n_nodes, fill=out_fill)
    got = out.cpu().numpy().astype(np.float64)
    assert (np.abs(got - ref) <= bound(host, q, tk, tv, parent, n_nodes, ref)).all()
    # the append: its rows and nothing else
    path = np.full((B, N), -1, np.int32)
    n_path = np.array([min(N, 3), 1, 0], np.int32)
    for bb in range(B):
        path[bb, :n_path[bb]] = np.arange(n_path[bb])
    b.ngc_commit_draft(dc, dev[1], dev[2], torch.as_tensor(path).cuda(), torch.as_tensor(n_path).cuda(), status=st)
    k2, v2 = planes_i16(dc)
    for bb in range(B):
        new = slice(so[bb] + lens[bb], so[bb] + lens[bb] + n_path[bb])
        for a, before, tree in ((k2, k1, tk), (v2, v1, tv)):
            want = before.copy()[:, :, so[bb]:so[bb + 1]]
            want[:, :, lens[bb]:lens[bb] + n_path[bb]] = tree[:, bb, :, :n_path[bb]].view(torch.int16).numpy()
            assert np.array_equal(a[:, :, so[bb]:so[bb + 1]], want), (bb, new)
    assert_guards(bufs)
    # the fork: alive rows of sequence 0 to the others, rows behind them as they were
    b.ngc_fork_kv(dc, torch.tensor([-1, 0, 0], dtype=torch.int32).cuda(), status=st)
    k3, v3 = planes_i16(dc)
    n0 = lens[0] + int(n_path[0])
    assert status_value(st) == 0 and dc.lens.tolist() == [n0] * 3
    for a, before in ((k3, k2), (v3, v2)):
        for bb in range(B):
            assert np.array_equal(a[:, :, so[bb]:so[bb] + n0], before[:, :, so[0]:so[0] + n0])
            assert np.array_equal(a[:, :, so[bb] + n0:so[bb + 1]], before[:, :, so[bb] + n0:so[bb + 1]])
    assert_guards(bufs)


@pytest.mark.parametrize("T", [40, 3000])
def test_canaries_behind_the_outputs_of_fp32_trees_and_of_the_verification(T):
    b = ngc()
    c, q, tk, tv, parent, _ = case(f32, 64, 4, 2, 1, [T], 5, "tree", seed=6)
    dc = device_cache(c)
    out, whole, fill = guarded(q.shape, f32)
    ws, ws_whole = guarded_workspace(b.workspace_bytes(b.OP_TREE_ATTN, dc, n_max=5))
    st = b.new_status()
    b.ngc_tree_attn(dc, q.cuda(), tk.cuda(), tv.cuda(), torch.as_tensor(parent).cuda(), out, ws=ws, status=st)
    assert status_value(st) == 0 and bool((whole[out.numel():] == fill).all()) and bool((ws_whole[ws.numel():] == 0xAB).all())
    tokens, par, p, q_d, u = draft_case(3, 7, 501, "tree", "draft", 2)
    outs = [guarded(s, torch.int32) for s in ((3, 7), (3,), (3,))]
    b.ngc_verify_draft(*[torch.as_tensor(x).cuda() for x in (tokens, par, p, u)], *[o[0] for o in outs], torch.as_tensor(q_d).cuda(), status=st)
    ref = draft.verify_draft(tokens, par, p, u, q_d)
    for (a, w, f), r in zip(outs, ref):
        assert np.array_equal(a.cpu().numpy(), r) and bool((w[a.numel():] == f).all())
    assert status_value(st) == 0


@pytest.mark.parametrize("mode", ["draft", "point", "greedy"])
@pytest.mark.parametrize("V", [1, 3, 130, 4099, 20000])
def test_verification_of_rows_at_any_alignment(V, mode):
    """Rows of 4-byte numbers that begin anywhere within 16 bytes, the draft's elsewhere than the target's; what lies before
    and behind them is NaN."""
    b = ngc()
    for seed, (a, e) in enumerate([(0, 0), (1, 1), (2, 3), (3, 0), (0, 2)]):
        tokens, par, p, q_d, u = draft_case(2, 6, V, "tree", mode, seed)
        ref = draft.verify_draft(tokens, par, p, u, q_d, greedy=mode == "greedy")

        def shifted(x, off):
            if x is None:
                return None
            whole = torch.full((x.size + 8,), float("nan"), device="cuda")
            whole[off:off + x.size] = torch.as_tensor(x).cuda().view(-1)
            return whole[off:off + x.size].view(x.shape)
        res = [torch.empty(s, dtype=torch.int32, device="cuda") for s in ((2, 6), (2,), (2,))]
        st = b.new_status()
        b.ngc_verify_draft(torch.as_tensor(tokens).cuda(), torch.as_tensor(par).cuda(), shifted(p, a), torch.as_tensor(u).cuda(), *res,
                           shifted(q_d, e), greedy=int(mode == "greedy"), status=st)
        assert status_value(st) == 0 and not ref[3].any()
        for x, r in zip(res, ref):
            assert np.array_equal(x.cpu().numpy(), r)


CLUSTERS = [  # d, Hq, Hkv, N, lens, nodes per tree: units of at most 128 and of more rows, joined in clusters of 2, 4 and 8
    (128, 12, 2, 1, [512], None), (128, 12, 2, 16, [1900], None), (128, 2, 2, 128, [700, 64], [128, 3]), (64, 8, 2, 12, [500, 1, 0], [12, 7, 1]),
    (128, 12, 2, 40, [600], None), (128, 28, 4, 33, [1000, 130], [33, 0]), (64, 4, 1, 70, [900], None), (128, 16, 1, 50, [1000], [49]),
    (128, 40, 2, 20, [257], None), (128, 1, 1, 1, [449, 0, 63, 64, 65], None)]


@pytest.mark.parametrize("d,Hq,Hkv,N,lens,nodes", CLUSTERS)
def test_short_units_joined_in_clusters(d, Hq, Hkv, N, lens, nodes):
    b = ngc()
    c, q, tk, tv, parent, n_nodes = case(bf16, d, Hq, Hkv, 1, lens, N, "tree", seed=N, n_nodes=nodes)
    assert b.tree_attn_launches(device_cache(c), N) == 1
    t_draft.check_tree(c, q, tk, tv, parent, n_nodes)
    t_draft.check_tree(c, q, tk, tv, parent, n_nodes, out_dtype=bf16)
    # a bad link and a bad length are reported and leave their sequence's rows alone, whichever CTA of the cluster meets them
    B = len(lens)
    bad = np.concatenate([parent, parent]), torch.cat([q, q], 1), torch.cat([tk, tk], 1), torch.cat([tv, tv], 1)
    two = synth.make_cache(1, 2 * B, Hq, Hkv, d, bf16, list(lens) * 2, capacity=max(lens), seed=3)
    n2 = None if nodes is None else np.concatenate([n_nodes, n_nodes])
    good, st = run_tree(two, *bad[1:], bad[0], n2)
    assert st == 0
    p2 = bad[0].copy()
    p2[B, 0] = 0
    out, st = run_tree(two, *bad[1:], p2, n2)
    assert st == 8 and (out[:, B] == -7).all()
    out[:, B] = good[:, B]
    assert torch.equal(out, good)
    ln = two.lens.clone()
    ln[0] = max(lens) + 1
    out, st = run_tree(two, *bad[1:], bad[0], n2, lens=ln)
    assert st == 1 and (out[:, 0] == -7).all()
    out[:, 0] = good[:, 0]
    assert torch.equal(out, good)


# ------------------------------------------------------------------ two calls at once

def test_calls_on_two_streams_at_once():
    """Each stream has its outputs, workspace and status: ten rounds of both at once give what each gives alone."""
    b = ngc()
    jobs = []
    for seed, (dtype, d, Hq, N, lens) in enumerate([(bf16, 128, 12, 40, [4000, 100, 900]), (bf16, 128, 12, 6, [2000] * 70), (f32, 64, 4, 6, [900, 1500])]):
        c, q, tk, tv, parent, _ = case(dtype, d, Hq, 2, 1, lens, N, "tree", seed=seed)
        dc, st = device_cache(c), b.new_status()
        dev = [x.cuda() for x in (q, tk, tv, torch.as_tensor(parent))]
        out = torch.zeros(q.shape, dtype=f32, device="cuda")
        ws = b.alloc_workspace(b.workspace_bytes(b.OP_TREE_ATTN, dc, n_max=N))
        v = [torch.as_tensor(x).cuda() for x in draft_case(20, 9, 5000, "tree", "draft", seed)]
        res = [torch.empty(s, dtype=torch.int32, device="cuda") for s in ((20, 9), (20,), (20,))]

        def run(dc=dc, dev=dev, out=out, ws=ws, st=st, v=v, res=res):
            b.ngc_tree_attn(dc, *dev, out, ws=ws, status=st)
            b.ngc_verify_draft(v[0], v[1], v[2], v[4], *res, v[3], status=st)
        run()
        jobs.append((run, torch.cuda.Stream(), [out] + res, [x.clone() for x in [out] + res], st))
    torch.cuda.synchronize()
    for _ in range(10):
        for _, _, got, _, _ in jobs:
            for x in got:
                x.zero_()
        for _, s, _, _, _ in jobs:
            s.wait_stream(torch.cuda.current_stream())
        for run, s, _, _, _ in jobs:
            with torch.cuda.stream(s):
                run()
        for _, s, _, _, _ in jobs:
            torch.cuda.current_stream().wait_stream(s)
        for _, _, got, want, st in jobs:
            assert status_value(st) == 0 and all(torch.equal(x, w) for x, w in zip(got, want))


@pytest.mark.parametrize("d,Hq,Hkv,N,B,T", [(128, 12, 2, 6, 70, 2000), (64, 12, 2, 6, 70, 2000), (128, 12, 2, 40, 30, 2010), (128, 2, 2, 3, 400, 450)])
def test_rows_are_the_same_whether_the_cache_comes_from_memory_or_l2(d, Hq, Hkv, N, B, T):
    """Late loads change the order in which the kernel's warps meet, not the result: runs behind a flushed L2 and warm ones agree
    to the bit, with one another and, within the bound, with the oracle (first and last sequence)."""
    b = ngc()
    lens = [T - i % 7 for i in range(B)]
    c, q, tk, tv, parent, _ = case(bf16, d, Hq, Hkv, 1, lens, N, "tree", seed=13)
    dc, st = device_cache(c), b.new_status()
    dev = [x.cuda() for x in (q, tk, tv, torch.as_tensor(parent))]
    ws = b.alloc_workspace(b.workspace_bytes(b.OP_TREE_ATTN, dc, n_max=N))
    flush = torch.empty(1 << 28, dtype=torch.uint8, device="cuda")
    outs = []
    for i in range(16):
        out = torch.zeros(q.shape, dtype=f32, device="cuda")
        if i % 4 < 3:
            flush.fill_(i)
        b.ngc_tree_attn(dc, *dev, out, ws=ws, status=st)
        outs.append(out)
    assert status_value(st) == 0 and all(torch.equal(x, outs[0]) for x in outs)
    for s in (0, B - 1):
        so = c.seq_off.numpy()
        one = synth.Cache(c.k[:, :, so[s]:so[s + 1]].contiguous(), c.v[:, :, so[s]:so[s + 1]].contiguous(), torch.tensor([0, int(so[s + 1] - so[s])]),
                          c.lens[s:s + 1], 1, 1, Hq, Hkv, d)
        x = [t[:, s:s + 1].contiguous() for t in (q, tk, tv)]
        ref = draft.tree_attn(synth.to_numpy(one.k), synth.to_numpy(one.v), one.seq_off.numpy(), one.lens.numpy(), *[synth.to_numpy(t) for t in x], parent[s:s + 1])
        assert (np.abs(outs[0][:, s:s + 1].cpu().numpy() - ref) <= bound(one, *x, parent[s:s + 1], None, ref)).all()


# ------------------------------------------------------------------ edges of the number range

KINDS = [(bf16, 128, 5, 600), (bf16, 128, 100, 900), (f32, 64, 5, 40), (f32, 64, 5, 3000), (f32, 128, 40, 3000), (bf16, 128, 5, 40), (bf16, 128, 5, 4000), (bf16, 128, 100, 4000), (bf16, 64, 5, 4000),
         (bf16, 128, 5, 14000), (bf16, 128, 100, 14000), (bf16, 64, 5, 14000)]


@pytest.mark.parametrize("dtype,d,N,T", KINDS)      # with one part per row and with several
def test_a_query_of_nan_gives_nan_and_changes_no_other_row(dtype, d, N, T):
    c, q, tk, tv, parent, _ = case(dtype, d, 4, 2, 1, [T, T], N, "tree", seed=7)
    clean, _ = run_tree(c, q, tk, tv, parent, None)
    q2 = q.clone()
    q2[0, 1, 2, 1, 3] = float("nan")
    out, st = run_tree(c, q2, tk, tv, parent, None)
    assert st == 0 and torch.isnan(out[0, 1, 2, 1]).all()
    out[0, 1, 2, 1] = clean[0, 1, 2, 1]
    assert torch.equal(out, clean)


@pytest.mark.parametrize("dtype,d,N,T", KINDS)
def test_scores_of_minus_infinity(dtype, d, N, T):
    """Where all that a row sees scores minus infinity its softmax is 0 / 0, a NaN; where some of it does, that has weight 0."""
    c, q, tk, tv, parent, _ = case(dtype, d, 4, 2, 1, [T], N, "tree", seed=9)
    q[..., 0] = 1.0
    c.k[..., 0] = float("-inf")
    empty = c.clone()
    empty.lens = torch.zeros_like(c.lens)
    ref = draft.tree_attn(synth.to_numpy(empty.k), synth.to_numpy(empty.v), c.seq_off.numpy(), empty.lens.numpy(), synth.to_numpy(q),
                          synth.to_numpy(tk), synth.to_numpy(tv), parent)
    out, st = run_tree(c, q, tk, tv, parent, None)
    assert st == 0 and (np.abs(out.cpu().numpy() - ref) <= bound(empty, q, tk, tv, parent, None, ref)).all()
    tk[..., 0] = float("-inf")
    out, st = run_tree(c, q, tk, tv, parent, None)
    assert st == 0 and torch.isnan(out).all()


@pytest.mark.parametrize("dtype,d,N,T", KINDS)
def test_scores_up_to_the_documented_size(dtype, d, N, T):
    """One cache row scores 2^29, everything else at most 2^28: its weight is 1, all others are 0.  Its weight is rounded once
    before the product (2^-8 on bf16 caches), the sum it is divided by is not; 1 / sum and the product are rounded in fp32
    (the two together, and an exponential that is the same on both sides, below 2^-20)."""
    c, q, tk, tv, _, _ = case(dtype, d, 4, 2, 1, [T], N, "tree", seed=11)
    parent = trees(1, N, "star", 0)
    q.zero_(); c.k.zero_(); tk.zero_()
    q[..., 0] = 2.0 ** 15
    c.k[..., 0] = torch.as_tensor(np.random.default_rng(0).integers(-128, 129, tuple(c.k.shape[:3]))).to(dtype) * 64      # exact, up to 2^13
    tk[..., 0] = 2.0 ** 13
    top = T // 2 + 1
    c.k[:, :, top, 0] = 2.0 ** 14
    out, st = run_tree(c, q, tk, tv, parent, None, scale=1.0)
    want = c.v[0, :, top].double().numpy()[None, None, :, None, None].repeat(2, 3).repeat(N, 4).reshape(1, 1, 4, N, d)
    assert st == 0 and (np.abs(out.double().cpu().numpy() - want) <= (2.0 ** -8 if dtype == bf16 else 2.0 ** -20) * np.abs(want) + 1e-30).all()
