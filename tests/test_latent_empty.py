"""Replay calls on batches without a single row: nothing to do, and no tensor that has an address."""
import ctypes as C

import pytest

from test_latent_limits import ngc, seqs      # noqa: F401


@pytest.mark.parametrize("R,max_len", [(0, 0), (0, 60), (2, 60)])
def test_calls_without_rows_do_nothing(ngc, R, max_len):      # noqa: F811
    s = seqs(ngc, rows=0, max_len=max_len)
    hist = (None, None, None, 0, 0) if R == 0 else (16, 16, 16, R, 4)
    head = [C.byref(s), None, None, None, *hist, 0, 0.1, None, 1, None]
    ws = 256 if R else None                                                   # (a history's workspace goes by max_len)
    n = ngc.lib.ngc_latent_replay_workspace_bytes(C.byref(s), 0, R, 1)
    assert (n > 0) == (R > 0)
    assert ngc.lib.ngc_latent_replay_attn(*head, ws, n, None, None) == 0
    assert ngc.lib.ngc_latent_replay_attn_backward(*head, None, None, None, None, ws, n, None, None) == 0
    head[10] = float("nan")                                                   # what else is wrong is refused all the same
    assert ngc.lib.ngc_latent_replay_attn(*head, ws, n, None, None) == -1
