"""Pins of the paged oracle against the dense one and by hand."""
import numpy as np
import pytest

import oracle


def test_pages_of_one_sequence_are_the_dense_forward():
    g = np.random.default_rng(1)
    L, D, page = 37, 8, 5
    q, k, v = g.standard_normal((2, L, D)), g.standard_normal((1, L, D)), g.standard_normal((1, L, D))
    ids = g.permutation(11)[:8]
    kp, vp = np.full((11, 1, page, D), np.nan), np.full((11, 1, page, D), np.nan)
    for j in range(L):
        kp[ids[j // page], 0, j % page], vp[ids[j // page], 0, j % page] = k[0, j], v[0, j]
    for mask in (dict(), dict(sinks=3), dict(sinks=2, units=True)):
        want, wl = oracle.attn_fwd(q[None], k[None], v[None], 3, 4, **mask)
        out, lse, add = oracle.paged_attn(q[:, 30:], kp, vp, [ids], [L], [0, 7], 3, 4, weigh=2, **mask)
        assert np.allclose(out, want[0, :, 30:]) and np.allclose(lse, wl[0, :, 30:])
        assert np.isclose(add[0].sum(), 2 * 2)  # two rows of two heads, each row's weights sum to one


def test_rows_that_see_nothing():
    kp = np.ones((2, 1, 4, 8))
    out, lse, add = oracle.paged_attn(np.ones((1, 3, 8)), kp, kp, [[0], [7]], [1, 4], [0, 2, 3], 4, 100, weigh=5)
    assert (out[0, 0] == 0).all() and lse[0, 0] == -np.inf     # position -1
    assert (out[0, 1] == 1).all()                              # position 0
    assert (out[0, 2] == 0).all() and lse[0, 2] == -np.inf     # its page is not there
    assert add[0].tolist() == [[1.0]] and (add[1] == 0).all()


@pytest.mark.parametrize("w,keep,sinks,recent,want", [
    ([1, 5, 3, 5, 2], 2, 0, 0, [1, 3]),
    ([1, 5, 3, 5, 2], 1, 0, 0, [1]),                 # ties: the lower row
    ([1, 5, 3, 5, 2], 3, 1, 1, [0, 1, 4]),
    ([1, 5, 3, 5, 2], 2, 2, 2, [0, 1]),              # more protected than kept: the lower rows
    ([float("nan"), -1.0, 0.0, float("-inf")], 3, 0, 0, [1, 2, 3]),
    ([0.0, -0.0, 0.0], 2, 0, 0, [0, 1]),
    ([1, 2], 0, 0, 0, []), ([1, 2], 9, 0, 0, [0, 1]),
])
def test_selection_by_hand(w, keep, sinks, recent, want):
    assert oracle.paged_select(np.array(w, dtype=np.float64), keep, sinks, recent).tolist() == want
