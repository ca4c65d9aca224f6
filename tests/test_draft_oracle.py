"""Drafted-token calls without a GPU: pins of the CPU oracle (against the one-token decode oracle, against a
sequence of appends, and against the distribution that verification must reproduce) and refusals on the host."""
import ctypes as C

import numpy as np
import pytest
import torch

import oracle
from oracle import draft
from paper_2604_18002_b200 import synth

bf16, f32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def ngc():
    from paper_2604_18002_b200 import build
    build.build()
    from paper_2604_18002_b200 import binding
    return binding


@pytest.mark.parametrize("dtype,d,Hq,Hkv", [(f32, 64, 4, 2), (bf16, 128, 6, 2)])
def test_chain_is_a_sequence_of_decode_appends(dtype, d, Hq, Hkv):
    L, B, N, lens = 2, 2, 4, [9, 0]
    c = synth.make_cache(L, B, Hq, Hkv, d, dtype, lens, capacity=16, seed=1)
    q, tk, tv = (synth.normal((L, B, H, N, d), s, dtype) for H, s in ((Hq, 2), (Hkv, 3), (Hkv, 4)))
    parent = np.tile(np.arange(-1, N - 1, dtype=np.int32), (B, 1))
    so = c.seq_off.numpy()
    k, v, ln = synth.to_numpy(c.k).copy(), synth.to_numpy(c.v).copy(), c.lens.numpy().copy()
    got = draft.tree_attn(k, v, so, ln, synth.to_numpy(q), synth.to_numpy(tk), synth.to_numpy(tv), parent)
    path = np.tile(np.arange(N, dtype=np.int32), (B, 1))
    k2, v2, ln2, st = draft.commit_draft(k, v, so, ln, synth.to_numpy(tk), synth.to_numpy(tv), path, np.full(B, N, np.int32))
    for i in range(N):
        ref, rc = oracle.decode_attn(k, v, so, ln, synth.to_numpy(q[:, :, :, i]), synth.to_numpy(tk[:, :, :, i]), synth.to_numpy(tv[:, :, :, i]))
        assert rc == 0 and np.allclose(got[:, :, :, i], ref, rtol=1e-10, atol=1e-12)
    assert not st.any() and np.array_equal(ln, ln2)
    for b in range(B):                      # rows beyond the lengths differ by nothing either: both left them alone
        assert np.array_equal(k[:, :, so[b]:so[b + 1]], k2[:, :, so[b]:so[b + 1]])
        assert np.array_equal(v[:, :, so[b]:so[b + 1]], v2[:, :, so[b]:so[b + 1]])


def test_branches_do_not_see_each_other():
    L, B, H, d, N = 1, 1, 1, 64, 5
    c = synth.make_cache(L, B, H, H, d, f32, [3], capacity=3, seed=1)
    q, tk, tv = (synth.normal((L, B, H, N, d), s, f32).numpy() for s in (2, 3, 4))
    parent = np.array([[-1, 0, 0, 1, 2]], np.int32)
    args = (c.k.numpy(), c.v.numpy(), c.seq_off.numpy(), c.lens.numpy())
    one = draft.tree_attn(*args, q, tk, tv, parent)
    tk2, tv2 = tk.copy(), tv.copy()
    tk2[..., 1, :] = np.inf                 # node 1: seen by nodes 1 and 3 only
    tv2[..., 1, :] = np.nan
    two = draft.tree_attn(*args, q, tk2, tv2, parent)
    assert np.array_equal(one[..., [0, 2, 4], :], two[..., [0, 2, 4], :]) and np.isnan(two[..., [1, 3], :]).all()


@pytest.mark.parametrize("kind", ["draft", "point"])
def test_verification_reproduces_the_target_distribution(kind):
    """The token after the root (an accepted child's, else the final draw) must be distributed as the target's row.
    20000 trials: a share is off by more than 5 standard deviations, sqrt(p (1 - p) / trials), with odds below 1e-6 a token."""
    V, trials, kids = 6, 20000, 3
    rng = np.random.default_rng(5)
    p = rng.dirichlet(np.ones(V)).astype(np.float32)
    q = rng.dirichlet(np.ones(V)).astype(np.float32)
    N = kids + 1
    parent = np.tile(np.array([-1] + [0] * kids, np.int32), (trials, 1))
    tokens = np.zeros((trials, N), np.int32)
    if kind == "draft":
        tokens[:, 1:] = rng.choice(V, (trials, kids), p=q.astype(np.float64) / q.astype(np.float64).sum())
    else:
        tokens[:, 1:] = np.argsort(-q)[:kids]
    target = np.broadcast_to(p, (trials, N, V))
    dr = np.broadcast_to(q, (trials, N, V)) if kind == "draft" else None
    u = rng.random((trials, N)).astype(np.float32)
    path, n_path, nxt, st = draft.verify_draft(tokens, parent, target, u, dr)
    assert not st.any()
    first = np.where(n_path > 1, tokens[np.arange(trials), np.maximum(path[:, 1], 0)], nxt)
    share = np.bincount(first, minlength=V) / trials
    assert np.all(np.abs(share - p) <= 5 * np.sqrt(p * (1 - p) / trials))
    assert 0.02 < (n_path > 1).mean() < 0.98                                  # both outcomes were exercised


def test_refusals_on_the_host(ngc):
    lib = ngc.lib
    good = ngc.CacheDesc(16, 16, 16, 16, 64, 2, 1, 12, 2, 128, ngc.BF16, 64)
    f32c = ngc.CacheDesc(16, 16, 16, 16, 64, 2, 1, 4, 4, 64, ngc.F32, 64)

    def tree(c, q=16, tk=16, tv=16, parent=16, N=4, lo=0, hi=2, scale=0.1, out=16, dt=ngc.F32, ws=None, nws=0):
        return lib.ngc_tree_attn(C.byref(c), q, tk, tv, parent, None, N, lo, hi, scale, out, dt, ws, nws, None, None)
    assert tree(good, q=None) == -1 and tree(good, tk=None) == -1 and tree(good, parent=None) == -1 and tree(good, out=None) == -1
    assert tree(good, q=24) == -1 and tree(good, out=8) == -1                       # not 16-byte aligned
    assert tree(good, N=0) == -1 and tree(good, N=129) == -2
    assert tree(good, lo=1, hi=1) == -1 and tree(good, hi=3) == -1 and tree(good, lo=-1) == -1
    for scale in (0.0, -1.0, float("nan"), float("inf")):
        assert tree(good, scale=scale) == -1
    assert tree(f32c, dt=ngc.BF16) == -1 and tree(good, dt=2) == -1
    long = ngc.CacheDesc(16, 16, 16, 16, 1 << 20, 2, 1, 12, 2, 128, ngc.BF16, 1 << 20)
    need = ngc.lib.ngc_workspace_bytes(ngc.OP_TREE_ATTN, C.byref(long), 1, 4, 0)
    assert need > 0 and need % 256 == 0 and tree(long) == -3 and tree(long, ws=256, nws=16) == -3
    assert ngc.lib.ngc_workspace_bytes(ngc.OP_TREE_ATTN, C.byref(long), 1, 129, 0) == 0
    assert lib.ngc_tree_attn(None, 16, 16, 16, 16, None, 4, 0, 2, 0.1, 16, 0, None, 0, None, None) == -1
    # paged: bf16, d = 128; pages of 32 or 64
    pg = ngc.PagedCacheDesc(16, 16, 16, 16, 1, 1, 12, 2, 128, ngc.BF16, 48, 4, 0)
    assert lib.ngc_tree_attn_paged(C.byref(pg), 16, 16, 16, 16, None, 4, 0, 1, 0.1, 16, 0, None, 0, None, None) == -1
    assert lib.ngc_commit_draft_paged(C.byref(pg), 16, 16, 16, 16, 4, None, None) == -1
    pg = ngc.PagedCacheDesc(16, 16, 16, 16, 1, 1, 4, 4, 64, ngc.F32, 32, 4, 0)
    assert lib.ngc_tree_attn_paged(C.byref(pg), 16, 16, 16, 16, None, 4, 0, 1, 0.1, 16, 0, None, 0, None, None) == -2
    assert lib.ngc_commit_draft_paged(C.byref(pg), 16, 16, 16, 16, 4, None, None) == -2
    assert lib.ngc_fork_pages(C.byref(pg), 16, None, None) == -2

    def verify(tok=16, par=16, p=16, q=16, u=16, B=2, N=4, V=100, greedy=0, path=16, n=16, nxt=16):
        return lib.ngc_verify_draft(tok, par, None, p, q, u, B, N, V, greedy, path, n, nxt, None, None)
    for kw in (dict(tok=None), dict(par=None), dict(p=None), dict(u=None), dict(path=None), dict(n=None), dict(nxt=None),
               dict(B=0), dict(N=0), dict(V=0)):
        assert verify(**kw) == -1
    assert verify(N=129) == -2
    assert lib.ngc_commit_draft(C.byref(good), None, 16, 16, 16, 4, None, None) == -1
    assert lib.ngc_commit_draft(C.byref(good), 16, 24, 16, 16, 4, None, None) == -1
    assert lib.ngc_commit_draft(C.byref(good), 16, 16, 16, 16, 0, None, None) == -1
    assert lib.ngc_commit_draft(C.byref(good), 16, 16, 16, 16, 129, None, None) == -2
    assert lib.ngc_commit_draft(None, 16, 16, 16, 16, 4, None, None) == -1
    assert lib.ngc_fork_kv(C.byref(good), None, None, None) == -1 and lib.ngc_fork_kv(None, 16, None, None) == -1
    assert ngc.lib.ngc_tree_attn_launches(C.byref(good), 2, 4) == 1 and ngc.lib.ngc_tree_attn_launches(C.byref(long), 2, 4) == 2


def test_binding_refuses_wrong_shapes_types_and_host_tensors(ngc):
    L, B, Hq, Hkv, d, N = 1, 2, 4, 2, 64, 3
    k = torch.zeros((L, Hkv, 32, d))
    cache = ngc.NgcCache(k, k.clone(), torch.tensor([0, 16, 32]), torch.zeros(B, dtype=torch.int32), Hq, 16)
    q, tk = torch.zeros((L, B, Hq, N, d)), torch.zeros((L, B, Hkv, N, d))
    parent = torch.tensor([[-1, 0, 1]] * B, dtype=torch.int32)
    ok = dict(q=q, tree_k=tk, tree_v=tk.clone(), parent=parent, out=q.clone())
    with pytest.raises(ngc.NgcError, match="device tensors required"):
        ngc.ngc_tree_attn(cache, **ok)
    for bad in (dict(q=q[:, :, :, :2]), dict(tree_k=tk.to(bf16)), dict(parent=parent.long()), dict(out=q[0]), dict(n_nodes=torch.zeros(3, dtype=torch.int32)),
                dict(status=torch.zeros(2, dtype=torch.int32))):
        with pytest.raises(ngc.NgcError, match="must be"):
            ngc.ngc_tree_attn(cache, **{**ok, **bad})
    with pytest.raises(ngc.NgcError, match="must be"):
        ngc.ngc_commit_draft(cache, tk, tk, parent, torch.zeros(B + 1, dtype=torch.int32))
    with pytest.raises(ngc.NgcError, match="must be"):
        ngc.ngc_fork_kv(cache, torch.zeros(B, dtype=torch.int64))
    p = torch.zeros((B, N, 10))
    with pytest.raises(ngc.NgcError, match="must be"):
        ngc.ngc_verify_draft(parent, parent, p.double(), torch.zeros((B, N)), parent, parent[:, 0], parent[:, 0])
    with pytest.raises(ngc.NgcError, match="contiguous"):
        ngc.ngc_verify_draft(parent, parent, p.transpose(0, 1).contiguous().transpose(0, 1), torch.zeros((B, N)), parent,
                             torch.zeros(B, dtype=torch.int32), torch.zeros(B, dtype=torch.int32))


def test_limits_of_scale_and_vocabulary(ngc):
    """scale * log2(e) has to stay finite, and token indices a round of loads ahead of the last one have to stay in 32 bits."""
    lib = ngc.lib
    c = ngc.CacheDesc(16, 16, 16, 16, 64, 2, 1, 12, 2, 128, ngc.BF16, 64)
    assert lib.ngc_tree_attn(C.byref(c), 16, 16, 16, 16, None, 4, 0, 2, 2.5e38, 16, ngc.F32, None, 0, None, None) == -1
    assert lib.ngc_verify_draft(16, 16, None, 16, 16, 16, 2, 4, (1 << 30) + 1, 0, 16, 16, 16, None, None) == -2


@pytest.mark.parametrize("dtype,d,N", [("BF16", 128, 16), ("BF16", 128, 40), ("BF16", 64, 1), ("F32", 64, 4)])
def test_workspace_serves_every_smaller_max_len(ngc, dtype, d, N):
    """How a call is laid out depends on max_len in steps, its workspace must not: one sized for a cache serves the call that
    gives a smaller max_len (a call is refused with NGC_ERR_WORKSPACE, before anything is launched, if it has too little)."""
    import itertools
    for layers, B in itertools.product((1, 3), (1, 2, 7, 16, 20, 32, 48, 64, 150)):
        last = 0
        for T in range(0, 12000, 97):
            c = ngc.CacheDesc(16, 16, 16, 16, B * T, layers, B, 12, 2, d, getattr(ngc, dtype), T)
            need = ngc.lib.ngc_workspace_bytes(ngc.OP_TREE_ATTN, C.byref(c), 1, N, 0)
            assert need >= last, (layers, B, T)
            for n in range(1, layers + 1):
                assert ngc.lib.ngc_tree_attn_launches(C.byref(c), n, N) == 1 or need > 0
            last = need
