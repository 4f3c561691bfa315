"""Sizes at which the launches of the paged calls reach the limits of a grid (host side only, nothing is enqueued)."""
import pytest

from test_paged_abi import _layer, _lg, _map


@pytest.mark.parametrize("hq,hkv,batch", [(32, 8, 128), (8, 8, 256), (64, 4, 64)])
def test_steps_whose_join_would_pass_a_grid_are_not_split(hq, hkv, batch):
    """The launch that joins splits has a workgroup of 256 threads for 8 rows at head_dim 128, and a grid fewer than 2^32
    threads: from 2^27 rows on a step is not split, so that the largest workspace is that of 2^27 - 8 rows."""
    lg = _lg()
    m = _map(lg, batch=batch, max_pages=512, page_size=256)  # 131072 slots: rows are split whatever the step's size
    l = _layer(lg, n_q_heads=hq, n_kv_heads=hkv, page_size=256)
    last = ((1 << 27) - 8) // hq
    size = lg.lg_paged_attend_workspace(l, m, last, 131072)
    assert size == 4 * last * hq * 132 * 4  # four splits of 32768 slots
    assert lg.lg_paged_attend_workspace(l, m, last - 1, 131072) < size
    for total in (last + 1, last + 1000, 2 * last):
        assert lg.lg_paged_attend_workspace(l, m, total, 131072) == size, total
