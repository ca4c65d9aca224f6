"""Decode steps of a rollout loop that admits long prompts: a step's slots and rows are those of its own tokens."""
import numpy as np
import pytest
import torch

from helpers import ngc
from oracle import latent as ora
from test_gpu_latent import assert_within, bf16, host, normal

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("lists", [0, 1])
def test_steps_after_long_prompts_take_slots_and_rows_of_their_tokens_only(lists):
    """The same life with a slot tensor for every call and with one for the prompts: books, rows and outputs are the same."""
    from paper_2604_18002_b200.rollout import NgcLatentRollout
    b = ngc()
    L, B, H, dc, dr, page, cap = 2, 4, 8, 128, 32, 32, 60
    prompt = [1500, 33, 700, 1025]
    max_new = sum(prompt) + 3
    ro = [NgcLatentRollout(L, B, H, dc, dr, 200, cap, max_new, 0.1, page, lists) for _ in range(2)]
    for r in ro:
        r.pool.rows.zero_()
    latent, rope = normal((L, max_new, dc), 1, 4).cuda(), normal((L, max_new, dr), 2).cuda()
    n_new = torch.tensor(prompt, dtype=torch.int32).cuda()
    for r in ro:
        r.update(n_new)
        r.write(latent, rope)
    for i, counts in enumerate([[1, 1, 1, 1], [1, 2, 0, 1], [1, -1, 1, 1], [1, 1, 1, 0]]):
        n_new = torch.tensor(counts, dtype=torch.int32).cuda()
        n = B if i % 2 else B + 5
        lat, rop = normal((L, n, dc), 10 + i, 4).cuda(), normal((L, n, dr), 20 + i).cuda()
        wide = [torch.full((L, max_new, w), float("nan"), dtype=bf16, device="cuda") for w in (dc, dr)]
        wide[0][:, :n], wide[1][:, :n] = lat, rop
        if i == 2:                                                             # a round, in which one rollout is left out
            units = -(-host(ro[0].pool.lens).max(1) // page)
            args = [torch.randn((B, ro[0].G, cap), generator=torch.Generator().manual_seed(3)).cuda(), torch.tensor(units, dtype=torch.int32).cuda(), None,
                    torch.tensor([20, -1, 9, 30], dtype=torch.int32).cuda(), 5, 0, n_new]
            ro[0].evict(*args, n_slots=n)
            ro[1].evict(*args)
        else:
            ro[0].update(n_new, n)
            ro[1].update(n_new)
        assert ro[0].slots.shape == (ro[0].G, n)
        ro[0].write(lat, rop)
        ro[1].write(*wide)
        assert torch.equal(ro[0].slots, ro[1].slots[:, :n]) and bool((ro[1].slots[:, n:] == -1).all()) and torch.equal(ro[0].first, ro[1].first)
        for x in ("page_table", "page_used", "lens", "rows"):
            assert torch.equal(getattr(ro[0].pool, x), getattr(ro[1].pool, x)), (i, x)
    ql, qr = normal((L, B, H, dc), 30), normal((L, B, H, dr), 31)
    out = torch.zeros((L, B, H, dc), device="cuda")
    ro[0].decode(ql.cuda(), qr.cuda(), out)
    for r in ro:
        r.check_status()
    want, bound = ora.decode(*[host(x) for x in (ro[0].pool.rows, ro[0].pool.page_table, ro[0].pool.lens)], host(ql), host(qr), 0.1, lists)
    assert_within(out, want, bound)


def test_too_few_slots_are_reported():
    from paper_2604_18002_b200.rollout import NgcLatentRollout
    b = ngc()
    ro = NgcLatentRollout(1, 3, 4, 128, 16, n_pages=20, pages_cap=4, max_new=100, scale=0.1, page=32)
    ro.update(torch.tensor([2, 1, 2], dtype=torch.int32).cuda(), 3)
    assert host(ro.pool.lens)[:, 0].tolist() == [2, 1, 0]
    with pytest.raises(b.NgcError, match="bad counts"):
        ro.check_status()
