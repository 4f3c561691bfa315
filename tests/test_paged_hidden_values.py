"""Values that a token does not see have no effect at all on it: whatever they are, its results are bit for bit those of
a run without them, since the weights of such slots are 0 exactly and so are their values in the products. A token
that sees an infinity or NaN in V gets it in that value alone."""
import numpy as np
import pytest
import torch

from test_parity_paged_attend import BF, F32, Attend

pytestmark = pytest.mark.gpu

COLUMN = 5


def _slot(a, b, j):
    return int(a.table_h[b, j // a.ps]), j % a.ps


def _run(a, dead, poisoned, keys, value):
    """Puts `value` where no slot is live, into one value of V of the slots (b, j), and, with keys, into one of K."""
    live = np.zeros((len(a.k), a.ps), bool)
    for b, n in enumerate(a.n):
        for j in range(a.have[b] + n):
            live[_slot(a, b, j)] = True
    if dead:
        rows = torch.as_tensor(~live, device="cuda")[:, None, :, None]
        a.k.masked_fill_(rows, value), a.v.masked_fill_(rows, value)
    for b, j in poisoned:
        p, row = _slot(a, b, j)
        a.v[p, :, row, COLUMN] = value
        if keys:
            a.k[p, :, row, 9] = value
    a.call()
    return a.results()


def _seen(a, b, i, j):
    m = a.have[b] + i
    return j <= m and (not a.window or a.pos_h[b, j] > a.pos_h[b, m] - a.window or a.pos_h[b, j] < a.sinks)


# Slots seen by no token (behind the first tokens, outside every window), by some, and by a decoding sequence or not.
SHAPES = [
    (128, 6, 2, [90, 40, 0], [30, 1, 3], 25, 4, [(0, 30), (0, 110), (1, 10), (2, 2)]),
    (64, 4, 4, [100, 64], [70, 2], 40, 0, [(0, 20), (0, 100), (0, 150), (1, 65), (1, 3)]),
    (128, 8, 2, [900, 33], [1, 4], 300, 16, [(0, 100), (0, 590), (1, 36), (1, 34)]),      # few rows, splits
    (128, 4, 1, [500], [300], 120, 8, [(0, 60), (0, 450), (0, 799), (0, 500)]),           # many rows
]


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), float("-inf"), 3e38])
@pytest.mark.parametrize("keys", [False, True])
@pytest.mark.parametrize("D,hq,hkv,have,n,window,sinks,poisoned", SHAPES)
def test_unseen_values_have_no_effect(dtype, value, keys, D, hq, hkv, have, n, window, sinks, poisoned):
    make = lambda: Attend(dtype, D, hq, hkv, 16, have, n, window=window, sinks=sinks, seed=11, holes=False, cap_pages=60)  # noqa: E731
    clean = make()
    clean.call()
    want, a = clean.results(), make()
    got = _run(a, True, poisoned, keys, value)
    hit = np.zeros(a.T, bool)
    for b, j in poisoned:
        for i in range(n[b]):
            hit[a.start_h[b] + i] |= _seen(a, b, i, j)
    assert hit.any() and not hit.all()
    for x, y in zip(want[:3], got[:3]):
        np.testing.assert_array_equal(x[~hit], y[~hit])
    for b in range(len(n)):
        if not hit[a.start_h[b + 1] - 1]:
            assert want[3][b] == got[3][b]


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("D,hq,hkv,have,n,window,sinks,poisoned", SHAPES)
def test_seen_values_reach_their_column_alone(dtype, value, D, hq, hkv, have, n, window, sinks, poisoned):
    make = lambda: Attend(dtype, D, hq, hkv, 16, have, n, window=window, sinks=sinks, seed=12, holes=False, gain=0.5,  # noqa: E731
                          cap_pages=60)
    clean = make()
    clean.call()
    want, a = clean.results(), make()
    got = _run(a, False, poisoned, False, value)
    hit = np.zeros(a.T, bool)
    for b, j in poisoned:
        for i in range(n[b]):
            hit[a.start_h[b] + i] |= _seen(a, b, i, j)
    assert hit.any() and not hit.all()
    for x, y in zip(want[1:], got[1:]):
        np.testing.assert_array_equal(x, y)
    np.testing.assert_array_equal(np.delete(want[0], COLUMN, 2), np.delete(got[0], COLUMN, 2))
    np.testing.assert_array_equal(want[0][~hit], got[0][~hit])
    reached = got[0][hit][:, :, COLUMN]
    assert np.isnan(reached).all() if np.isnan(value) else (reached == value).all()
