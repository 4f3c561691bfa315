"""The softmax weights of the few-row forms of lg_paged_attend (decode steps, few new tokens a sequence, beside long
chunks too) enter the product with bfloat16 V as two terms, like those of lg_decode_attend.

The inputs leave only the weights' precision to see. A key and a query have one value each that is not 0, so a score is
one exact product, at most 2 / sqrt(D); the slots come in pairs whose scores are one bfloat16 step apart and whose
values are opposite, so that outputs nearly cancel and their own rounding is small. Error bound, relative to
sum alpha |v|: 2^-16 for the two terms, and in units of 2^-24: 8 for the argument and result of an exponential,
and one for each of the additions in a row, to the sum of weights (at most n / 4 + 32 and the joins, at most 80) and
to the output (twice as many); then half a step of the result, 2^-8 of it."""
import numpy as np
import pytest
import torch

from oracle import paged
from test_parity_paged_attend import BF, Attend

pytestmark = pytest.mark.gpu


def _pairs(a, seed):
    """One value a query and key; pairs of slots with neighbouring keys and opposite values."""
    r = np.random.RandomState(seed)
    a.q.zero_(), a.k.zero_(), a.v.zero_()
    a.q[:, :, 0] = 1.0
    for b, n in enumerate(a.n):
        m = a.have[b] + n
        order = r.permutation(m)[:m // 2 * 2].reshape(2, -1)
        low = 1 + r.randint(0, 127, (order.shape[1], a.hkv)) / 128  # in [1, 2): bfloat16 steps of 1 / 128
        u = torch.as_tensor(r.randn(order.shape[1], a.hkv, a.D), device="cuda").to(BF)
        for side in (0, 1):
            page = a.i32(a.table_h[b, order[side] // a.ps]).long()
            row = a.i32(order[side] % a.ps).long()
            a.k[page, :, row, 0] = torch.as_tensor(low + side / 128, device="cuda").to(BF)
            a.v[page, :, row] = u if side == 0 else -u


@pytest.mark.parametrize("D,hq,hkv,have,n", [
    (128, 28, 4, [37, 90, 3, 200], [1, 1, 1, 1]),            # splits
    (128, 8, 2, [700, 33], [1, 1]),
    (128, 8, 4, [40 + 3 * b for b in range(16)], [1] * 16),  # two workgroups share a row's outputs
    (128, 8, 8, [20 + b for b in range(40)], [1] * 40),      # one workgroup a row
    (64, 16, 1, [60, 128, 5], [2, 1, 2]),                    # 32 and 16 rows
    (64, 4, 4, [50, 90], [20, 3]),
    (128, 8, 2, [45, 80, 61], [40, 1, 3]),                   # beside a chunk of 160 rows
    (64, 8, 2, [100, 80, 61], [100, 1, 8]),
])
def test_weights_of_few_rows(D, hq, hkv, have, n):
    a = Attend(BF, D, hq, hkv, 16, have, n, seed=D + hq + len(n), holes=False)
    _pairs(a, seed=hq)
    a.call()
    out = a.results()[0]
    k, v, q = (x.double().cpu().numpy() for x in (a.k, a.v, a.q))
    G, looked = hq // hkv, 0
    for b in range(len(n)):
        if n[b] * G > 32:
            continue  # a long chunk
        slots = np.arange(have[b] + n[b])
        page = a.table_h[b, slots // 16]
        rows = np.arange(a.start_h[b], a.start_h[b] + n[b])
        for h in range(hkv):
            want, _, _, av, _ = paged.attend(q[rows, h * G:(h + 1) * G], k[page, h, slots % 16], v[page, h, slots % 16],
                                             slots, have[b], 0, 0, 0)
            depth = len(slots) / 4 + 32 + 80
            tol = (2.0 ** -16 + (3 * depth + 8) * 2.0 ** -24) * av * (1 + 2.0 ** -8) + 2.0 ** -8 * np.abs(want)
            got = out[rows, h * G:(h + 1) * G]
            assert (np.abs(got - want) <= tol).all(), (b, h, (np.abs(got - want) / tol).max())
            looked += 1
    assert looked


@pytest.mark.parametrize("value", [float("inf"), float("-inf")])
@pytest.mark.parametrize("D,hq,hkv,have,n", [(128, 8, 4, [100] * 16, [1] * 16), (64, 16, 1, [300], [2]), (128, 4, 2, [90, 64], [80, 1])])
def test_infinite_values_of_exact_weights(D, hq, hkv, have, n, value):
    """Weights that are bfloat16 numbers themselves (all scores are 0) leave no term of 0 for an infinity to meet, in
    tiles that every row sees and in others."""
    a = Attend(BF, D, hq, hkv, 16, have, n, seed=3, holes=False)
    a.q.zero_()
    for b in range(len(n)):
        for slot, dim in ((5, 3), (have[b] - 1, 7)):
            a.v[int(a.table_h[b, slot // 16]), :, slot % 16, dim] = value
    a.call()
    out = a.results()[0][:a.start_h[-1]]
    assert (out[:, :, [3, 7]] == value).all()
    assert np.isfinite(np.delete(out, [3, 7], 2)).all()
