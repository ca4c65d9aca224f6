"""The rollout loop of latent attention without a GPU: what it refuses before a call."""
import pytest
import torch


@pytest.fixture(scope="module")
def ngc():
    from paper_2604_18002_b200 import build
    build.build()
    from paper_2604_18002_b200 import binding
    return binding


def test_slots_of_a_call_are_some_of_the_rollouts(ngc):
    from paper_2604_18002_b200.rollout import NgcLatentRollout
    ro = NgcLatentRollout(2, 3, 4, 128, 16, n_pages=8, pages_cap=4, max_new=90, scale=0.1, page=32, lists=ngc.LISTS_PER_LAYER, device="cpu")
    n_new, i32 = torch.ones(3, dtype=torch.int32), torch.int32
    for n in (0, -1, 91):
        with pytest.raises(ngc.NgcError, match="n_slots"):
            ro.update(n_new, n)
        with pytest.raises(ngc.NgcError, match="n_slots"):
            ro.evict(torch.zeros((3, 2, 4)), n_new, None, n_new, 1, 0, n_new, n_slots=n)
    assert ro.slots.shape == (2, 90)
    for n in (3, 1, None, 90, 3):
        with pytest.raises(ngc.NgcError, match="device tensors"):             # the arguments are right, the library has no CPU path
            ro.update(n_new, n)
        assert ro.slots.shape == (2, n or 90) and ro.slots.is_contiguous() and ro.slots.data_ptr() == ro._all_slots.data_ptr()
    bf = torch.bfloat16
    with pytest.raises(ngc.NgcError, match="latent"):
        ro.write(torch.zeros((2, 90, 128), dtype=bf), torch.zeros((2, 90, 16), dtype=bf))
    with pytest.raises(ngc.NgcError, match="device tensors"):
        ro.write(torch.zeros((2, 3, 128), dtype=bf), torch.zeros((2, 3, 16), dtype=bf))
