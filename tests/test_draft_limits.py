"""Drafted-token calls without a GPU: what the oracle and the host refuse at the edges."""
import ctypes as C

import numpy as np
import pytest

from oracle import draft


@pytest.mark.parametrize("drafted", [False, True])
def test_oracle_wants_probabilities_where_a_child_is_tested(drafted):
    """A chain whose only child is accepted whatever its probability: its row is never summed."""
    p = np.full((1, 2, 4), 0.25, np.float32)
    tokens, parent, u = np.array([[0, 2]], np.int32), np.array([[-1, 0]], np.int32), np.zeros((1, 2), np.float32)
    for x, status in ((0.25, 0), (1e-30, 0), (-0.25, 9), (np.inf, 9), (-np.inf, 9), (np.nan, 9)):
        for r in ("p", "q") if drafted else ("p",):
            p2, q2 = p.copy(), p.copy()
            (p2 if r == "p" else q2)[0, 0, 2] = x
            path, n_path, nxt, st = draft.verify_draft(tokens, parent, p2, u, q2 if drafted else None)
            assert st.tolist() == [status] and n_path.tolist() == ([2] if status == 0 else [0])
            assert path.tolist() == ([[0, 1]] if status == 0 else [[-1, -1]]) and (nxt[0] >= 0) == (status == 0)


def test_calls_whose_tiles_pass_32_bits_are_refused():
    """The tiles of a call, with what stands for the beginning of a unit, are counted in 32 bits on the device.  300 million strips
    would pass that; 100 million, or ones whose rows are as many as a plane can have, do not."""
    from paper_2604_18002_b200 import build
    build.build()
    from paper_2604_18002_b200 import binding as ngc

    def launches(B, Hq, Hkv, N, d, rows, max_len, L=1, layers=1, dtype=ngc.BF16):
        c = ngc.CacheDesc(16, 16, 16, 16, rows, L, B, Hq, Hkv, d, dtype, max_len)
        return ngc.lib.ngc_tree_attn_launches(C.byref(c), layers, N)
    assert launches(300_000_000, 1, 1, 1, 64, 300_000_000, 1) == 0
    assert launches(150_000_000, 2, 2, 1, 64, 150_000_000, 1) == 0
    assert launches(50_000_000, 1, 1, 1, 64, 0, 0, L=6, layers=6) == 0
    assert launches(100_000_000, 1, 1, 1, 64, 100_000_000, 1) == 1
    assert launches(1, 1, 1, 1, 64, 0x7fffffff, 0x7fffffff) == 2
    assert launches(4, 28, 4, 33, 128, 0x7fffffff, 0x7fffffff, L=4, layers=4) > 0
    c = ngc.CacheDesc(16, 16, 16, 16, 300_000_000, 1, 300_000_000, 1, 1, 64, ngc.BF16, 1)
    assert ngc.lib.ngc_tree_attn(C.byref(c), 16, 16, 16, 16, None, 1, 0, 1, 0.1, 16, ngc.F32, None, 0, None, None) == -2
