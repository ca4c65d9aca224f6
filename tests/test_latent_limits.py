"""Latent-attention calls without a GPU: what the host refuses before anything is launched, and workspace sizes."""
import ctypes as C

import pytest
import torch


@pytest.fixture(scope="module")
def ngc():
    from paper_2604_18002_b200 import build
    build.build()
    from paper_2604_18002_b200 import binding
    return binding


def pool(ngc, L=2, B=3, dc=512, dr=64, dtype=1, page=64, cap=8, n_pages=20, lists=1, rows=16, table=16, used=16, lens=16):
    return ngc.LatentPoolDesc(rows, table, used, lens, L, B, dc, dr, dtype, page, cap, n_pages, lists)


def seqs(ngc, off=16, lens=16, rows=100, L=1, B=2, H=4, dn=128, dv=128, dr=64, dtype=1, max_len=60):
    return ngc.LatentSeqsDesc(off, lens, rows, L, B, H, dn, dv, dr, dtype, max_len)


def test_structs_match_the_header(ngc):
    assert C.sizeof(ngc.LatentPoolDesc) == 72 and ngc.LatentPoolDesc.L.offset == 32 and ngc.LatentPoolDesc.lists.offset == 64
    assert C.sizeof(ngc.LatentSeqsDesc) == 56 and ngc.LatentSeqsDesc.rows.offset == 16 and ngc.LatentSeqsDesc.max_len.offset == 52


BAD_POOLS = [dict(L=0), dict(B=0), dict(page=16), dict(page=128), dict(cap=0), dict(n_pages=0), dict(lists=3), dict(lists=-1), dict(rows=None),
             dict(table=None), dict(used=None), dict(lens=None), dict(dtype=2), dict(dr=0), dict(L=40000, n_pages=2000)]


@pytest.mark.parametrize("bad", BAD_POOLS)
def test_calls_on_a_pool_that_is_none_are_refused(ngc, bad):
    c = C.byref(pool(ngc, **bad))
    assert ngc.lib.ngc_pool_update(c, None, None, 0, 16, 16, 4, 16, None, None) == -1
    assert ngc.lib.ngc_latent_write(c, 16, 4, 16, 16, 0, 1, None, None) == -1
    assert ngc.lib.ngc_latent_decode(c, 16, 16, 8, 0, 1, 0.1, 16, 0, 256, 1 << 40, None, None) == -1


def test_arguments_of_pool_update_and_write_are_refused(ngc):
    lib, c = ngc.lib, C.byref(pool(ngc))
    assert lib.ngc_pool_update(None, None, None, 0, 16, 16, 4, 16, None, None) == -1
    for kept, budget, k_max, n_new, slots, n_slots, first in [(16, None, 4, 16, 16, 4, 16), (None, 16, 4, 16, 16, 4, 16), (16, 16, 0, 16, 16, 4, 16),
                                                             (None, None, 0, None, 16, 4, 16), (None, None, 0, 16, None, 4, 16),
                                                             (None, None, 0, 16, 16, 0, 16), (None, None, 0, 16, 16, 4, None)]:
        assert lib.ngc_pool_update(c, kept, budget, k_max, n_new, slots, n_slots, first, None, None) == -1
    assert lib.ngc_pool_update(C.byref(pool(ngc, B=8193)), None, None, 0, 16, 16, 4, 16, None, None) == -2
    assert lib.ngc_pool_update(c, None, None, 0, 16, 16, 2 ** 30, 16, None, None) == -2
    for args in [(None, 4, 16, 16, 0, 1), (16, 0, 16, 16, 0, 1), (16, 4, None, 16, 0, 1), (16, 4, 16, None, 0, 1), (16, 4, 16, 16, 1, 1), (16, 4, 16, 16, -1, 1),
                 (16, 4, 16, 16, 0, 3), (16, 4, 24, 16, 0, 1), (16, 4, 16, 20, 0, 1)]:
        assert lib.ngc_latent_write(c, *args, None, None) == -1
    for bad in (dict(dtype=0), dict(dc=96), dict(dc=640), dict(dr=8), dict(dr=72), dict(dr=80)):
        assert lib.ngc_latent_write(C.byref(pool(ngc, **bad)), 16, 4, 16, 16, 0, 1, None, None) == -2


def test_arguments_of_decode_are_refused(ngc):
    lib, p = ngc.lib, pool(ngc)
    c, need = C.byref(p), ngc.lib.ngc_latent_decode_workspace_bytes(C.byref(p), 16)
    ok = dict(ql=16, qr=16, H=16, lo=0, hi=1, scale=0.1, out=16, dt=0, ws=256, n=need)

    def call(c=c, **kw):
        a = dict(ok, **kw)
        return lib.ngc_latent_decode(c, a["ql"], a["qr"], a["H"], a["lo"], a["hi"], a["scale"], a["out"], a["dt"], a["ws"], a["n"], None, None)
    for kw in (dict(ql=None), dict(qr=None), dict(out=None), dict(H=0), dict(lo=1), dict(lo=-1), dict(hi=3), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")),
               dict(scale=float("inf")), dict(scale=3e38), dict(dt=2), dict(ql=24), dict(qr=8), dict(out=20)):
        assert call(**kw) == -1, kw
    assert call(H=129) == -2 and call(C.byref(pool(ngc, dtype=0))) == -2 and call(C.byref(pool(ngc, dc=320))) == -2 and call(C.byref(pool(ngc, dr=24))) == -2
    assert call(ws=None) == -3 and call(n=need - 1) == -3 and call(ws=128) == -3


def test_arguments_of_the_replay_calls_are_refused(ngc):
    lib, s = ngc.lib, seqs(ngc)
    need = lib.ngc_latent_replay_workspace_bytes(C.byref(s), 0, 2, 1)
    ok = dict(q=16, kv=16, kr=16, pos=16, count=16, total=16, R=2, kt=4, lists=0, scale=0.1, out=16, dt=1, lse=16, go=16, gq=16, gkv=16, gkr=16, ws=256, n=need)

    def call(back, s=s, **kw):
        a = dict(ok, **kw)
        head = [C.byref(s)] + [a[k] for k in ("q", "kv", "kr", "pos", "count", "total", "R", "kt", "lists", "scale", "out", "dt", "lse")]
        if not back:
            return lib.ngc_latent_replay_attn(*head, a["ws"], a["n"], None, None)
        return lib.ngc_latent_replay_attn_backward(*head, a["go"], a["gq"], a["gkv"], a["gkr"], a["ws"], a["n"], None, None)
    for back in (False, True):
        for kw in (dict(q=None), dict(kv=None), dict(kr=None), dict(out=None), dict(pos=None), dict(count=None), dict(total=None), dict(R=-1), dict(kt=0), dict(lists=3),
                   dict(scale=0.0), dict(scale=float("nan")), dict(dt=3), dict(q=8), dict(kv=24), dict(kr=4), dict(out=8)):
            assert call(back, **kw) == -1, kw
        for bad in (dict(off=None), dict(lens=None), dict(rows=-1), dict(L=0), dict(B=0), dict(H=0), dict(max_len=-1)):
            assert call(back, seqs(ngc, **bad)) == -1, bad
        for bad in (dict(dn=64), dict(dv=64), dict(dr=8), dict(dr=80), dict(dtype=0), dict(rows=2 ** 31, L=1), dict(rows=2 ** 30, L=3), dict(L=300, B=300)):
            assert call(back, seqs(ngc, **bad)) == -2, bad
        assert call(back, ws=None) == -3 and call(back, ws=128) == -3 and call(back, n=(need if back else 512) - 1) == -3
    for kw in (dict(lse=None), dict(go=None), dict(gq=None), dict(gkv=None), dict(gkr=None), dict(go=8), dict(gq=4), dict(gkv=12), dict(gkr=8)):
        assert call(True, **kw) == -1, kw


def test_workspace_sizes(ngc):
    lib = ngc.lib
    for H, heads in ((1, 16), (16, 16), (17, 32), (40, 64), (128, 128)):
        n = lib.ngc_latent_decode_workspace_bytes(C.byref(pool(ngc)), H)
        assert n % 256 == 0 and n >= 2 * (148 // (2 if H > 64 else 1)) * heads * 512 * 4
        assert n == lib.ngc_latent_decode_workspace_bytes(C.byref(pool(ngc, L=1, B=7000, n_pages=5, cap=100)), H)
    s = C.byref(seqs(ngc))
    assert lib.ngc_latent_replay_workspace_bytes(s, 0, 0, 0) == 0                     # causal: none
    assert lib.ngc_latent_replay_workspace_bytes(s, 0, 3, 0) == 1024 + 256            # 2 x 128 tokens, 2 x 1 tiles
    assert lib.ngc_latent_replay_workspace_bytes(s, 0, 0, 1) == 1792 + 100 * 4 * 64 * 4
    assert lib.ngc_latent_decode_workspace_bytes(None, 4) == 0 and lib.ngc_latent_replay_workspace_bytes(None, 0, 1, 1) == 0


def test_tensors_of_the_host_or_of_other_shapes_are_refused(ngc):
    p = ngc.new_latent_pool(2, 3, 128, 16, 10, 4, page=32, lists=1, device="cpu")
    i32 = torch.int32
    with pytest.raises(ngc.NgcError, match="device tensors"):
        ngc.ngc_pool_update(p, torch.zeros(3, dtype=i32), torch.zeros((2, 5), dtype=i32), torch.zeros(4, dtype=i32))
    with pytest.raises(ngc.NgcError, match="n_new"):
        ngc.ngc_pool_update(p, torch.zeros(4, dtype=i32), torch.zeros((2, 5), dtype=i32), torch.zeros(4, dtype=i32))
    with pytest.raises(ngc.NgcError, match="slots"):
        ngc.ngc_pool_update(p, torch.zeros(3, dtype=i32), torch.zeros((1, 5), dtype=i32), torch.zeros(4, dtype=i32))
    with pytest.raises(ngc.NgcError, match="kept_sorted"):
        ngc.ngc_pool_update(p, torch.zeros(3, dtype=i32), torch.zeros((2, 5), dtype=i32), torch.zeros(4, dtype=i32), torch.zeros((3, 1, 2), dtype=i32), torch.zeros(3, dtype=i32))
    bf = torch.bfloat16
    with pytest.raises(ngc.NgcError, match="rope"):
        ngc.ngc_latent_write(p, torch.zeros((2, 5), dtype=i32), torch.zeros((2, 5, 128), dtype=bf), torch.zeros((2, 5, 32), dtype=bf))
    with pytest.raises(ngc.NgcError, match="q_latent"):
        ngc.ngc_latent_decode(p, torch.zeros((2, 3, 4, 64), dtype=bf), torch.zeros((2, 3, 4, 16), dtype=bf), torch.zeros((2, 3, 4, 128), dtype=bf), 0.1)
    with pytest.raises(ngc.NgcError, match="contiguous"):
        ngc.ngc_latent_decode(p, torch.zeros((2, 3, 128, 4), dtype=bf).transpose(2, 3), torch.zeros((2, 3, 4, 16), dtype=bf), torch.zeros((2, 3, 4, 128), dtype=bf), 0.1)
    p.lens = p.lens.long()
    with pytest.raises(ngc.NgcError, match="lens"):
        ngc.latent_decode_workspace_bytes(p, 4)
    s = ngc.NgcLatentSeqs(torch.tensor([0, 10]), torch.tensor([10], dtype=i32), 10)
    q, kv, kr, out = (torch.zeros(x, dtype=bf) for x in ((1, 10, 2, 160), (1, 10, 2, 256), (1, 10, 32), (1, 10, 2, 128)))
    with pytest.raises(ngc.NgcError, match="device tensors"):
        ngc.ngc_latent_replay_attn(s, q, kv, kr, out)
    with pytest.raises(ngc.NgcError, match="kv"):
        ngc.ngc_latent_replay_attn(s, q, kv[:, :, :, :128].contiguous(), kr, out)
    with pytest.raises(ngc.NgcError, match="k_rope"):
        ngc.ngc_latent_replay_attn(s, q, kv, torch.zeros((1, 10, 64), dtype=bf), out)
    with pytest.raises(ngc.NgcError, match="alive_count"):
        ngc.ngc_latent_replay_attn(s, q, kv, kr, out, None, torch.zeros((2, 1, 1, 4), dtype=i32), torch.zeros((2, 1), dtype=i32), torch.zeros((2, 1), dtype=i32))
    with pytest.raises(ngc.NgcError, match="grad_k_rope"):
        ngc.ngc_latent_replay_attn_backward(s, q, kv, kr, out, torch.zeros((1, 2, 10)), out, q, kv, q)
