"""Drafted-token calls where their parts meet: units that follow one another in a CTA, parts that a second kernel joins,
draws and rows at the edge of what counts as a probability."""
import numpy as np
import pytest
import torch

from helpers import ngc, status_value
from oracle import draft
from paper_2604_18002_b200 import synth
from test_gpu_draft import bound, case, check_verify, device_cache, draft_case, run_tree, run_verify

pytestmark = pytest.mark.gpu

bf16, f32 = torch.bfloat16, torch.float32


# ------------------------------------------------------------------ tree attention: from one unit to the next

@pytest.mark.parametrize("d,Hq,Hkv,N,B,first,launches", [
    (128, 2, 1, 80, 600, "refused", 1), (128, 2, 1, 80, 600, "one node", 1), (64, 2, 1, 80, 600, "refused", 1), (128, 4, 1, 96, 400, "refused", 1),
    (128, 4, 2, 70, 300, "refused", 1), (128, 2, 1, 128, 600, "one node", 1), (128, 3, 1, 100, 250, "refused", 1), (128, 2, 1, 80, 200, "refused", 2),
    (128, 2, 1, 80, 200, "one node", 2)])
def test_empty_caches_behind_trees_that_leave_early(d, Hq, Hkv, N, B, first, launches):
    """More than 128 query rows per KV head, units dealt out whole (one launch) or cut (two): every other sequence leaves its unit
    early (its tree is refused, or has one node), the one behind it has an empty cache, so that its first tile is a tree tile whose
    V rows are mended at once.  The softmax groups of the two M tiles are then as far apart as they get.  Runs behind a flushed L2
    and warm ones agree to the bit, and with the oracle within the bound."""
    b = ngc()
    lens = [0 if i % 2 else (300, 129, 0, 260)[i // 2 % 4] for i in range(B)]
    n_nodes = np.full(B, N, np.int32)
    c, q, tk, tv, parent, _ = case(bf16, d, Hq, Hkv, 1, lens, N, "tree", seed=N, capacity=300)
    if first == "refused":
        parent[::2, N - 1] = N - 1
    else:
        n_nodes[::2] = 1
    dc, st = device_cache(c), b.new_status()
    assert b.tree_attn_launches(dc, N) == launches
    dev = [x.cuda() for x in (q, tk, tv, torch.as_tensor(parent))]
    dn = torch.as_tensor(n_nodes).cuda()
    ws = b.alloc_workspace(b.workspace_bytes(b.OP_TREE_ATTN, dc, n_max=N))
    flush = torch.empty(1 << 28, dtype=torch.uint8, device="cuda")
    outs = []
    for i in range(12):
        out = torch.full(q.shape, -7.0, dtype=f32, device="cuda")
        if i % 2:
            flush.fill_(i)
        st.zero_()
        b.ngc_tree_attn(dc, *dev, out, dn, ws=ws, status=st)
        assert status_value(st) == (8 if first == "refused" else 0)
        outs.append(out)
    assert all(torch.equal(x, outs[0]) for x in outs)
    ref = draft.tree_attn(synth.to_numpy(c.k), synth.to_numpy(c.v), c.seq_off.numpy(), c.lens.numpy(), *[synth.to_numpy(x) for x in (q, tk, tv)],
                          parent, n_nodes, fill=-7.0)
    got = outs[0].cpu().numpy().astype(np.float64)
    assert (got[ref == -7.0] == -7.0).all() and (np.abs(got - ref) <= bound(c, q, tk, tv, parent, n_nodes, ref)).all()


# ------------------------------------------------------------------ verification: the final draw

@pytest.mark.parametrize("o", [0, 3 * 16384 + 5 * 2048])
@pytest.mark.parametrize("drafted", [False, True])
def test_a_token_without_mass_is_never_drawn(o, drafted):
    """The draw's target, 1 / 8, is exactly the sum of the tokens before a run of the scan (token o), and the run's own sum is the
    double before its exact tie with that: 1 / 8 + (1 / 8 + 3 * 2^-55) rounds up, so that the run seems to begin 2^-55 beyond
    the target.  Its first token has no mass; the token drawn is the first one that has."""
    V, b = 131072, ngc()
    p = np.zeros((1, 1, V), np.float32)
    p[0, 0, [o, o + 9, o + 10, 131000]] = 0.125, 0.125, 3 * 2.0 ** -55, 0.75
    u, none = np.full((1, 1), 0.125, np.float32), np.array([[-1]], np.int32)
    ref = draft.verify_draft(none, none, p, u, p if drafted else None)
    assert ref[2].tolist() == [o + 9] and not ref[3].any()
    path, n_path, nxt, st = run_verify(none, none, p, u, p if drafted else None)
    assert st == 0 and path.tolist() == [[0]] and n_path.tolist() == [1] and nxt.tolist() == [o + 9]


# ------------------------------------------------------------------ verification: probabilities that are none

@pytest.mark.parametrize("mode", ["draft", "point"])
def test_a_tested_child_needs_probabilities(mode):
    """A tree whose walk tests children at two nodes and leaves both behind; in the second sequence one of the numbers that a test
    needs is negative, infinite or NaN, at nodes whose rows are not summed (or, where a drawn child is refused, not all of them).
    Elsewhere in the first node's row nobody looks."""
    V, N = 300, 6
    tokens, _, p, q, u = draft_case(3, N, V, "chain", mode, 5)
    parent = np.tile(np.array([-1, 0, 0, 1, 1, 4], np.int32), (3, 1))      # walk: 0, 1 (2 is not tested), 4 (behind 3), 5
    tokens[:] = np.arange(N) + 7
    p[:, 1, tokens[0, 3]] = 0.0                                           # node 3 is refused, node 4 taken
    u[:, 1:] = 0.0
    u[:, 3] = 0.5
    if mode == "point":
        q = None
    else:
        q[:, 1] = p[:, 1]                                                 # what is left after node 3: p - q would be nothing, so it stays
        q[:, 1, tokens[0, 3]] = 0.25
    good = check_verify(tokens, parent, p, q, u)
    assert good[0][0].tolist() == [0, 1, 4, 5, -1, -1]
    for at, child in ((0, 1), (1, 3), (1, 4)):
        for rows in ("p", "q") if mode == "draft" else ("p",):
            for x in (-0.25, np.inf, -np.inf, np.nan):
                p2, q2 = p.copy(), None if q is None else q.copy()
                (p2 if rows == "p" else q2)[1, at, tokens[1, child]] = x
                ref = check_verify(tokens, parent, p2, q2, u)
                assert ref[3].tolist() == [0, 9, 0] and ref[2][1] == -1 and ref[1][1] == 0, (at, child, rows, x)
    p2 = p.copy()
    p2[1, 0, 200] = np.nan                                                # node 0's row is read at one token only
    ref = check_verify(tokens, parent, p2, q, u)
    assert not ref[3].any() and np.array_equal(ref[0], good[0])


# ------------------------------------------------------------------ tree attention: CTAs of a call

def kernel_grids(call):
    """Grid sizes of the kernels that a call enqueues, from its capture."""
    from cuda.bindings import driver
    graph = torch.cuda.CUDAGraph(keep_graph=True)
    with torch.cuda.graph(graph):
        call()

    def good(res):
        assert res[0] == driver.CUresult.CUDA_SUCCESS
        return res[1:]
    raw = driver.CUgraph(graph.raw_cuda_graph())
    nodes = good(driver.cuGraphGetNodes(raw, good(driver.cuGraphGetNodes(raw))[1]))[0]
    params = [good(driver.cuGraphKernelNodeGetParams(x))[0] for x in nodes]
    return [x.gridDimX * x.gridDimY * x.gridDimZ for x in params]


@pytest.mark.parametrize("N,T", [(1, 64), (16, 128), (1, 1), (70, 130)])
@pytest.mark.parametrize("B", [148, 149, 200, 296, 600])
def test_many_short_units_use_every_sm(B, N, T):
    """A unit (one KV head of a sequence) is work for a CTA however short it is: with 148 units and more all 148 SMs get some."""
    b = ngc()
    c, q, tk, tv, parent, _ = case(bf16, 128, 2, 1, 1, [T] * B, N, "tree", seed=1)
    dc, st = device_cache(c), b.new_status()
    dev = [x.cuda() for x in (q, tk, tv, torch.as_tensor(parent))]
    out = torch.zeros(q.shape, dtype=f32, device="cuda")
    ws = b.alloc_workspace(b.workspace_bytes(b.OP_TREE_ATTN, dc, n_max=N))

    def call():
        b.ngc_tree_attn(dc, *dev, out, ws=ws, status=st)
    call()
    grids = kernel_grids(call)
    assert len(grids) == b.tree_attn_launches(dc, N) and grids[0] >= 148 and status_value(st) == 0


# ------------------------------------------------------------------ tree attention: units that are cut and joined by a second kernel

CUT = [  # d, Hq, Hkv, N, lens: few long sequences, many units, one and two M tiles
    (128, 12, 2, 6, [16100, 900]), (64, 12, 2, 6, [20000]), (128, 12, 2, 40, [13000, 70]), (128, 4, 2, 16, [700 - 7 * i % 300 for i in range(80)]),
    (128, 4, 2, 70, [300 - 11 * i % 300 for i in range(80)])]


def cut_job(d, Hq, Hkv, N, lens, seed=0):
    """A call that cuts its units, with outputs, workspace and status of its own."""
    b = ngc()
    c, q, tk, tv, parent, _ = case(bf16, d, Hq, Hkv, 1, lens, N, "tree", seed=seed)
    dc, st = device_cache(c), b.new_status()
    assert b.tree_attn_launches(dc, N) == 2
    dev = [x.cuda() for x in (q, tk, tv, torch.as_tensor(parent))]
    out = torch.zeros(q.shape, dtype=f32, device="cuda")
    ws = b.alloc_workspace(b.workspace_bytes(b.OP_TREE_ATTN, dc, n_max=N))

    def run(ws=ws):
        b.ngc_tree_attn(dc, *dev, out, ws=ws, status=st)
    return run, out, st, dev, ws, (c, q, tk, tv, parent)


def within_bound(out, c, q, tk, tv, parent, n_nodes=None):
    ref = draft.tree_attn(synth.to_numpy(c.k), synth.to_numpy(c.v), c.seq_off.numpy(), c.lens.numpy(), *[synth.to_numpy(x) for x in (q, tk, tv)],
                          parent, n_nodes)
    return bool((np.abs(out.cpu().numpy() - ref) <= bound(c, q, tk, tv, parent, n_nodes, ref)).all())


def test_cut_calls_on_two_streams_at_once():
    jobs = [(cut_job(*x, seed=i), torch.cuda.Stream()) for i, x in enumerate(CUT)]
    want = []
    for (run, out, st, *_), _ in jobs:
        run()
        want.append(out.clone())
    torch.cuda.synchronize()
    for _ in range(10):
        for (run, out, *_), s in jobs:
            out.zero_()
            s.wait_stream(torch.cuda.current_stream())
        for (run, *_), s in jobs:
            with torch.cuda.stream(s):
                run()
                run()
        for _, s in jobs:
            torch.cuda.current_stream().wait_stream(s)
        for ((_, out, st, *_), _), w in zip(jobs, want):
            assert status_value(st) == 0 and torch.equal(out, w)


@pytest.mark.parametrize("i", range(len(CUT)))
def test_cut_calls_from_memory_and_from_l2(i):
    run, out, st, _, _, host = cut_job(*CUT[i], seed=20 + i)
    flush = torch.empty(1 << 28, dtype=torch.uint8, device="cuda")
    first = None
    for r in range(12):
        out.zero_()
        if r % 4 < 3:
            flush.fill_(r)
        run()
        first = out.clone() if first is None else first
        assert torch.equal(out, first)
    assert status_value(st) == 0 and within_bound(out, *host)


def test_cut_calls_in_graphs():
    """Two captured calls replay on new inputs: at once on two streams, each with its workspace; and, captured with one workspace
    between them, one after the other."""
    b = ngc()
    jobs = [cut_job(*CUT[i], seed=40 + i) for i in (0, 2)]
    shared = max((x[4] for x in jobs), key=lambda w: w.numel())
    graphs = []
    for run, *_ in jobs:
        run()
        for kw in ({}, dict(ws=shared)):
            graphs.append(torch.cuda.CUDAGraph())
            with torch.cuda.graph(graphs[-1]):
                run(**kw)
    side = torch.cuda.Stream()
    for seed in (1, 2):
        want = []
        for run, out, st, dev, _, _ in jobs:
            dev[0].copy_(synth.normal(dev[0].shape, seed, bf16))
            run()
            want.append(out.clone())
            out.zero_()
        side.wait_stream(torch.cuda.current_stream())
        graphs[0].replay()
        with torch.cuda.stream(side):
            graphs[2].replay()
        torch.cuda.current_stream().wait_stream(side)
        for (_, out, st, *_), w in zip(jobs, want):
            assert status_value(st) == 0 and torch.equal(out, w)
            out.zero_()
        graphs[1].replay()
        graphs[3].replay()
        for (_, out, st, *_), w in zip(jobs, want):
            assert status_value(st) == 0 and torch.equal(out, w)


@pytest.mark.parametrize("N,lens,max_len", [(16, [250, 0, 1, 64, 129, 300], 32768), (16, [250, 0, 1, 64, 129, 300] * 12, 8192), (70, [250, 0, 1, 64], 1 << 20),
                                            (1, [1], 1 << 20), (1, [0], 1 << 30), (40, [300] * 30, 8192)])
def test_lengths_far_below_max_len(N, lens, max_len):
    """A pruned cache: max_len says nothing about the lengths.  The plan cuts units that turn out to be short; most CTAs get none."""
    b = ngc()
    c, q, tk, tv, parent, _ = case(bf16, 128, 12, 2, 1, lens, N, "tree", seed=N)
    dc = device_cache(c)
    dc.max_len = max_len
    assert b.tree_attn_launches(dc, N) == 2
    out, st = run_tree(c, q, tk, tv, parent, None, max_len=max_len)
    assert st == 0 and within_bound(out, c, q, tk, tv, parent)
    none = np.zeros(len(lens), np.int32)
    out, st = run_tree(c, q, tk, tv, parent, none, max_len=max_len)                      # no tree has a node: no work at all
    assert st == 0 and (out == -7).all()


@pytest.mark.parametrize("drafted", [False, True])
@pytest.mark.parametrize("V", [5, 1000, 50001])
def test_negative_numbers_of_a_summed_row_count_as_zeros(V, drafted):
    """In the last node's row, of an only node and behind a refused child.  A row of nothing else has no positive sum."""
    for seed, (N, x) in enumerate([(1, -1e-6), (1, -3.0), (3, -1e-6), (3, -3.0), (3, -0.0)]):
        tokens, parent, p, q, u = draft_case(4, N, V, "star", "draft", 10 * V + seed)
        tokens[:, 1:] = 1
        u[:, 1:] = 1.0 - 2.0 ** -24
        q[:, :, 1] = 1.0                                      # u q(1) stays above p(1): every child is refused
        dr = q if drafted else None
        p[2, 0, V // 2:] = 0.0
        good = check_verify(tokens, parent, p, dr, u)
        assert (good[1] == 1).all() and not good[3].any()
        p2 = p.copy()
        p2[2, 0, V // 2:] = x
        ref = check_verify(tokens, parent, p2, dr, u)
        assert all(np.array_equal(a, r) for a, r in zip(ref, good))
        p2[2, 0] = x
        p2[2, 0, 1] = 0.0                                     # (of the refused child's token: it is tested)
        ref = check_verify(tokens, parent, p2, dr, u)
        assert ref[3].tolist() == [0, 0, 9, 0]
