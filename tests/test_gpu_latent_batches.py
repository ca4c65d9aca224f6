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
