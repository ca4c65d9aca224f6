"""Drafted-token calls without a GPU: what the oracle and the host refuse at the edges."""
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
