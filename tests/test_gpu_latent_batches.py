"""Latent attention of whole sequences in batches of thousands of short ones."""
import numpy as np
import pytest

from helpers import status_value
from test_gpu_latent import Replay, bf16

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("B,H,rounds,longest", [(1500, 2, None, 1), (2111, 1, [(0.5, 0.5)], 1), (1100, 3, [(0.3, 0.4), (0.8, 0.7)], 900)])
def test_batches_of_many_short_sequences(B, H, rounds, longest):
    """More sequences than a warp looks over at once, empty ones among them, and a long one at the end."""
    rng = np.random.default_rng(B)
    lens = [int(x) for x in rng.integers(0, 40, B)]
    lens[B // 3], lens[-1], lens[0] = 150, max(longest, lens[-1]), 0
    r = Replay(1, B, H, 32, lens, 1, 90, rounds)
    r.forward(bf16)
    r.check_forward()
    r.backward()
    r.check_backward()
    assert status_value(r.st) == 0


@pytest.mark.parametrize("rounds", [None, [(0.3, 0.5), (0.6, 0.5)]])
def test_a_bound_on_the_lengths_may_be_far_above_them(rounds):
    r = Replay(1, 3, 2, 64, [300, 1, 170], 2, 95, rounds)
    r.seqs.max_len = 70001
    r.forward(bf16)
    r.check_forward()
    r.backward()
    r.check_backward()
    assert status_value(r.st) == 0


def test_a_batch_without_rows():
    r = Replay(2, 2, 2, 64, [0, 0], 0, 96, None)
    r.seqs.max_len = 50
    assert r.forward(bf16)[0].numel() == 0
    assert all(g.numel() == 0 for g in r.backward())
    assert status_value(r.st) == 0
