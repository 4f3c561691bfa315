"""The suffix mass and confidence of lg_paged_attend where tiles begin with slots whose page is missing (bounds as in
test_parity_paged_attend.py)."""
import numpy as np
import pytest
import torch

from test_parity_paged_attend import BF, F32, Attend

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,D,hq,hkv", [(BF, 128, 8, 2), (BF, 64, 4, 4), (F32, 128, 4, 2), (F32, 64, 8, 1)])
@pytest.mark.parametrize("n", [1, 3, 50])
@pytest.mark.parametrize("window,sinks", [(0, 0), (70, 20)])
def test_suffix_behind_missing_pages(dtype, D, hq, hkv, n, window, sinks):
    """Pages of 16 slots in tiles of 32 or 64: the first page of a tile is missing, the others hold slots far older than
    the suffix."""
    a = Attend(dtype, D, hq, hkv, 16, [90, 20, 200], [n, 1, n], window=window, sinks=sinks, seed=n + D, suffix=[10, 3, 40])
    gone = {0: [0, 2], 1: [0], 2: [0, 4, 8]}
    for b, cols in gone.items():
        a.table_h[b, cols] = -1
        a.see[b] = ~np.isin(np.arange(a.have[b] + a.n[b]) // 16, cols)
    a.alloc()
    a.call()
    a.check()
