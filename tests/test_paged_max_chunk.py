"""max_chunk as a bound: a serving loop that captures its step gives the largest chunk it will ever bring, so decode
steps run in the form for long chunks (bounds as in test_parity_paged_attend.py)."""
import numpy as np
import pytest

from test_parity_paged_attend import BF, F32, Attend

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,D,hq,hkv", [(BF, 128, 28, 4), (BF, 64, 16, 1), (F32, 128, 4, 2), (F32, 64, 16, 1), (F32, 128, 16, 1)])
@pytest.mark.parametrize("chunk", [33, 2048, 2 ** 31 - 1])
@pytest.mark.parametrize("window,sinks", [(0, 0), (50, 4)])
def test_larger_than_the_step(dtype, D, hq, hkv, chunk, window, sinks):
    a = Attend(dtype, D, hq, hkv, 16, [0, 100, 333, 65, 7], [1, 1, 2, 0, 1], window=window, sinks=sinks, seed=D + hq)
    a.chunk = chunk
    a.alloc()
    a.call()
    a.check()


def test_nothing_allowed():
    """max_chunk 0: every sequence with tokens is refused."""
    a = Attend(BF, 64, 4, 2, 16, [20, 30, 5], [1, 2, 0], seed=1)
    a.chunk, a.skip = 0, {0, 1}
    a.alloc()
    a.call()
    a.check()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("first", [1, 5])
def test_rows_before_the_first_sequence(dtype, first):
    """q_start may begin behind row 0: rows before it belong to no sequence and stay as they are."""
    for n in ([1, 3, 1], [40, 1, 70]):
        a = Attend(dtype, 128, 4, 2, 16, [600, 33, 90], n, seed=first, extra=first + 2)
        a.start_h = a.start_h + first
        a.alloc()
        a.call()
        got = a.results()
        assert all((x[:first] == 7).all() for x in got[:3])
        a.check(got, tokens=np.array([0, 1, 33, -1]))


def test_one_of_the_statistics():
    """suffix_mass and conf are independent of each other."""
    for n in ([1, 2], [50, 1]):
        a, b, c = (Attend(BF, 128, 8, 2, 16, [700, 30], n, seed=4) for _ in range(3))
        a.call()
        for x, sm, conf in ((b, b.sm, None), (c, None, c.conf)):
            x.lg.lg_paged_attend(x.layer, x.map, x.q, x.out, x.q_start, x.base, x.chunk, 0, 0, x.sw, x.lse, sm, conf, x.ws)
        w, g, h = a.results(), b.results(), c.results()
        for i in (0, 1):
            np.testing.assert_array_equal(w[i], g[i]), np.testing.assert_array_equal(w[i], h[i])
        np.testing.assert_array_equal(w[2], g[2]), np.testing.assert_array_equal(w[3], h[3])
        assert (g[3] == 0.125).all() and (h[2] == 7).all()
