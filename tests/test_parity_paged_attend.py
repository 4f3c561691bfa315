"""lg_paged_attend against attention in 64 bits (oracle/paged.py), at the sizes, masks and values where it can
go wrong.

Error bounds. With S = max over the visible slots of sum_d |q_d k_d| / sqrt(D), a score is off by at most
(D + 4) 2^-24 S (a float32 sum of D exact products, the scaling), its exponential by that and 4 units of
2^-24, and the sum of n weights by (depth + 4 tiles) 2^-24, depth = 64 + n / 32 additions in a row and a
rescaling with each tile. So with
    e = ((D + 8) S + 2 n / 32 + 2 (64 + n / 32) + 16) 2^-24
the log of the sum is within e (+ 2^-22 of itself and of the largest score), a weight within 2 e of itself, and
out = sum alpha v within (2 e + w) sum alpha |v| + half a step of out, where w = 2^-8 is a bfloat16 layer's
rounding of each weight (0 in float32). Weights below 2^-126 of the row's largest are no normal float32 and
become 0, so a mass of n slots may be n 2^-126 short beside that."""
import numpy as np
import pytest
import torch

from oracle import paged

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32


class Attend:
    """A step: sequences of have[b] slots that bring n[b] tokens, pages in random order, holes in the positions."""

    def __init__(self, dtype, D, hq, hkv, ps, have, n, window=0, sinks=0, seed=0, extra=3, suffix=None, holes=True,
                 cap_pages=0, gain=2.0, table_gap=0):
        from paper_2604_10044_amd import lg
        self.lg, self.n, self.have, self.D, self.hq, self.hkv, self.ps, self.dtype = lg, n, have, D, hq, hkv, ps, dtype
        self.window, self.sinks = window, sinks
        self.r = r = np.random.RandomState(seed)
        B, P = len(n), max(cap_pages, max(-(-(h + x) // ps) for h, x in zip(have, n)))
        P = max(P, 1)
        self.P, n_pages = P, B * P + 5
        self.i32 = i32 = lambda x: torch.as_tensor(np.asarray(x, np.int32), device="cuda")  # noqa: E731
        self.table_h = r.permutation(n_pages)[:B * P].reshape(B, P)
        steps = np.where(r.rand(B, P * ps) < 0.2, r.randint(1, 9, (B, P * ps)), 1) if holes else np.ones((B, P * ps), int)
        self.pos_h = np.cumsum(steps, 1) - steps[:, :1] + (r.randint(0, 3, (B, 1)) if holes else 0)
        g = torch.Generator(device="cuda").manual_seed(seed)
        rand = lambda *s: torch.randn(*s, generator=g, device="cuda").to(dtype)  # noqa: E731
        self.k, self.v = rand(n_pages, hkv, ps, D), rand(n_pages, hkv, ps, D)
        self.T = sum(n) + extra
        self.q = (gain * rand(self.T, hq, D)).to(dtype)
        self.sw_h = np.asarray([max(1, (h + x) // 4) for h, x in zip(have, n)] if suffix is None else suffix)
        self.base_h = np.asarray(have)
        self.start_h = np.concatenate([[0], np.cumsum(n)])
        self.see = {}      # sequence -> slots that hold a page
        self.skip = set()  # refused sequences
        self.chunk = max(n) if len(n) else 1
        self.alloc()

    def alloc(self):
        lg = self.lg
        self.table, self.pos = self.i32(self.table_h), self.i32(self.pos_h)
        self.base, self.q_start, self.sw = self.i32(self.base_h), self.i32(self.start_h), self.i32(self.sw_h)
        self.len, self.ref = self.i32(self.base_h), self.i32(np.ones(len(self.k)))
        self.layer = lg.paged_layer(self.k, self.v, self.hq)
        self.map = lg.page_map(self.table, self.pos, self.len, self.ref, self.ps)
        self.out = torch.full_like(self.q, 7.0)
        self.lse = torch.full((self.T, self.hq), 7.0, device="cuda")
        self.sm = torch.full((self.T, self.hq), 7.0, device="cuda")
        self.conf = torch.full((len(self.n),), 0.125, device="cuda")
        size = lg.lg_paged_attend_workspace(self.layer, self.map, self.T, self.chunk)
        self.ws = torch.full((size,), 0xff, dtype=torch.uint8, device="cuda")  # NaN: nothing is read unwritten

    def call(self, stream=None, statistics=True):
        self.lg.lg_paged_attend(self.layer, self.map, self.q, self.out, self.q_start, self.base, self.chunk, self.window,
                                self.sinks, self.sw if statistics else None, self.lse, self.sm if statistics else None,
                                self.conf if statistics else None, self.ws, stream=stream)

    def results(self):
        torch.cuda.synchronize()
        return [x.double().cpu().numpy() for x in (self.out, self.lse, self.sm, self.conf)]

    def check(self, got=None, statistics=True, tokens=None):
        """tokens: rows to check where the sequences are long (all rows are checked for being written)."""
        out, lse, sm, conf = self.results() if got is None else got
        G, D, ps = self.hq // self.hkv, self.D, self.ps
        k, v, q = (x.double().cpu().numpy() for x in (self.k, self.v, self.q))
        for b, n in enumerate(self.n):
            rows = np.arange(self.start_h[b], self.start_h[b] + n)
            if b in self.skip:
                assert (out[rows] == 7).all() and (lse[rows] == 7).all() and (sm[rows] == 7).all()
                assert n == 0 or not statistics or np.isnan(conf[b])
                continue
            m = self.have[b] + n
            slots = np.arange(m)
            page = self.table_h[b, slots // ps]
            see = self.see.get(b)
            page = np.where((page >= 0) & (page < len(k)), page, 0)
            pos = self.pos_h[b, :m]
            pick = np.arange(n) if tokens is None or n == 0 else np.unique(np.clip(tokens, -n, n - 1) % max(n, 1))
            best = 0.0
            for h in range(self.hkv):
                kk, vv = k[page, h, slots % ps], v[page, h, slots % ps]
                for i in pick:
                    qq = q[rows[i], h * G:(h + 1) * G][None]
                    e = self.have[b] + i + 1
                    o, ls, ms, av, big = (x[0] for x in paged.attend(
                        qq, kk[:e], vv[:e], pos[:e], e - 1, self.window, self.sinks, int(self.sw_h[b]),
                        None if see is None else see[:e]))
                    got_o = out[rows[i], h * G:(h + 1) * G]
                    got_l, got_m = lse[rows[i], h * G:(h + 1) * G], sm[rows[i], h * G:(h + 1) * G]
                    err = ((D + 8) * big + 4 * e / 32 + 144) * 2.0 ** -24
                    half, w = (2.0 ** -8, 2.0 ** -8) if self.dtype is BF else (2.0 ** -24, 0.0)
                    tol = ((2 * err[:, None] + w) * av) * (1 + half) + half * np.abs(o)
                    what = (b, h, i)
                    empty = ~np.isfinite(ls)
                    assert (np.abs(got_o - o) <= tol).all(), (what, np.abs(got_o - o).max(), tol.min())
                    assert (got_l[empty] == -np.inf).all() and (got_o[empty] == 0).all(), what
                    ok = ~empty
                    assert (np.abs(got_l - ls)[ok] <= (err + 2.0 ** -22 * (np.abs(ls) + big))[ok]).all(), what
                    if statistics:
                        assert (np.abs(got_m - ms) <= 2 * err * ms + e * 2.0 ** -126).all(), (what, got_m, ms)
                    if i == n - 1:
                        best = max(best, got_m.max())
            if statistics and n and (n - 1) in pick:
                assert conf[b] == max(best, 0.125), (b, conf[b], best)
            elif n == 0:
                assert conf[b] == 0.125
        behind = self.start_h[-1]
        assert (out[behind:] == 7).all() and (lse[behind:] == 7).all()
        if statistics:
            assert (sm[behind:] == 7).all()
        else:
            assert (sm == 7).all() and (conf == 0.125).all()


SMALL = [
    # dtype, D, hq, hkv, page, have, n
    (BF, 128, 28, 4, 64, [0, 1, 63, 64, 65, 200], [1, 1, 1, 1, 1, 1]),       # a decode step
    (BF, 128, 28, 4, 16, [0, 5, 130, 31], [5, 4, 3, 0]),                     # 35, 28 and 21 rows: both shapes
    (BF, 64, 4, 4, 16, [0, 17, 3], [40, 33, 32]),                            # one query head a KV head
    (BF, 64, 16, 1, 32, [100, 0], [2, 3]),                                   # 16 a KV head: 32 and 48 rows
    (BF, 128, 32, 8, 128, [0, 127], [129, 2]),
    (BF, 128, 6, 2, 256, [250, 10], [70, 1]),
    (BF, 128, 5, 1, 16, [0], [77]),                                          # groups that straddle waves
    (F32, 64, 4, 4, 16, [160, 0], [16, 1]),
    (F32, 128, 8, 2, 32, [0, 45, 7], [33, 1, 9]),
    (F32, 64, 7, 1, 64, [0, 64], [5, 4]),
    (F32, 128, 16, 1, 16, [31, 0, 90], [1, 3, 0]),
]


@pytest.mark.parametrize("window,sinks", [(0, 0), (1, 0), (7, 4), (40, 20), (100000, 4)])
@pytest.mark.parametrize("dtype,D,hq,hkv,ps,have,n", SMALL)
def test_small(dtype, D, hq, hkv, ps, have, n, window, sinks):
    a = Attend(dtype, D, hq, hkv, ps, have, n, window=window, sinks=sinks, seed=D + hq + window)
    a.call()
    a.check()


@pytest.mark.parametrize("dtype,D,hq,hkv,ps,have,n,window,sinks", [
    (BF, 128, 12, 2, 16, [5000, 333], [1, 1], 0, 0),          # few rows: many splits, joined
    (BF, 128, 12, 2, 64, [9000], [1], 512, 32),               # the window skips most of the cache
    (BF, 64, 4, 4, 16, [4000], [64], 0, 0),                   # many rows, split
    (BF, 128, 28, 4, 64, [2000, 100, 1500], [1, 150, 20], 700, 32),
    (F32, 128, 8, 2, 16, [3000], [1], 0, 0),
    (F32, 64, 4, 1, 32, [1500, 0], [40, 300], 600, 4),
])
def test_long(dtype, D, hq, hkv, ps, have, n, window, sinks):
    a = Attend(dtype, D, hq, hkv, ps, have, n, window=window, sinks=sinks, seed=7)
    a.call()
    a.check(tokens=np.array([0, 1, 17, 63, 64, -1]))


@pytest.mark.parametrize("dtype,D,hq,hkv,batch", [
    (BF, 128, 4, 4, 32),    # 128 pairs: two workgroups share a row's outputs
    (BF, 128, 14, 2, 45),   # 90 pairs: the last group of 8 is short
    (BF, 128, 8, 1, 70),    # 70: three splits
    (F32, 128, 4, 2, 50),   # 100 pairs in float32
    (BF, 64, 16, 4, 32),
    (BF, 128, 8, 8, 40),    # 320: one workgroup each
])
def test_decode_batches(dtype, D, hq, hkv, batch):
    """A token a sequence at batch sizes that take each launch of the decode step."""
    have = [(37 * b) % 700 for b in range(batch)]
    a = Attend(dtype, D, hq, hkv, 16, have, [1] * batch, seed=batch)
    a.call()
    a.check()
    w = Attend(dtype, D, hq, hkv, 16, have, [1] * batch, window=100, sinks=5, seed=batch)
    w.call()
    w.check()


@pytest.mark.parametrize("dtype,D,hq,hkv,have,n", [
    (BF, 128, 8, 2, [950, 3, 500], [1, 1, 1]),         # few pairs: splits
    (BF, 128, 4, 1, [700], [8]),
    (BF, 128, 8, 2, [1100, 3, 500], [1, 1, 1]),
    (BF, 128, 8, 4, [1400] + [60] * 15, [1] * 16),     # 64 pairs: two workgroups share a row's outputs
    (F32, 128, 8, 2, [950, 3, 500], [1, 4, 4]),        # 16 rows
    (F32, 128, 8, 2, [950, 3, 500], [5, 1, 0]),        # 20
    (F32, 64, 16, 4, [300, 33], [8, 1]),               # 32
    (F32, 64, 16, 1, [300, 33], [1, 1]),               # 16
    (F32, 64, 5, 1, [40, 0], [6, 3]),                  # 30 and 15
    (F32, 128, 2, 1, [130] * 70, [16] + [9] * 69),     # 32 and 18, halves
    (F32, 128, 3, 3, [90] * 40, [16] + [1] * 39),      # 16 and 1, halves
])
def test_few_rows(dtype, D, hq, hkv, have, n):
    """Steps without long chunks at the edges of their launches: rows of a matrix instruction, halves and splits."""
    a = Attend(dtype, D, hq, hkv, 16, have, n, seed=sum(n) + D)
    a.call()
    a.check(tokens=np.array([0, 1, 3, 4, -1]))


def test_long_capacity():
    """More slots of capacity than a split may have: the launch splits rows though it has workgroups enough, and
    most splits are empty."""
    a = Attend(BF, 64, 32, 32, 256, [3, 700, 40, 0, 90, 2000, 31, 64, 5], [1, 1, 2, 1, 0, 1, 1, 40, 1], seed=23)
    more = 300 - a.P
    a.table_h = np.concatenate([a.table_h, np.full((9, more), -1)], 1)
    a.pos_h = np.concatenate([a.pos_h, np.full((9, more * 256), -1)], 1)
    assert 300 * 256 > 2 * 32768
    a.alloc()
    a.call()
    a.check(tokens=np.array([0, 1, 39]))


def test_long_prompt():
    """Thousands of tokens in one chunk behind others, two sequences."""
    a = Attend(BF, 128, 8, 2, 64, [1000, 3], [2100, 700], seed=8, holes=False)
    a.call()
    a.check(tokens=np.array([0, 1, 31, 32, 500, 1023, 1024, 2047, -2, -1]))


def test_large_offsets():
    """Pages whose bytes lie beyond 2^32."""
    from paper_2604_10044_amd import lg
    n_pages, ps, hkv, D = 70000, 128, 2, 128  # 4.6 GB each of K and V
    k = torch.zeros(n_pages, hkv, ps, D, dtype=BF, device="cuda")
    v = torch.zeros_like(k)
    a = Attend(BF, D, 4, hkv, ps, [200, 100], [3, 20], seed=9)
    pages = np.array([[69999, 5, 65535], [65536, 68000, 1]])[:, :a.P]
    for b in range(2):
        for c in range(a.P):
            k[int(pages[b, c])], v[int(pages[b, c])] = a.k[int(a.table_h[b, c])], a.v[int(a.table_h[b, c])]
    a.call()
    small = a.results()
    a.out.fill_(7), a.lse.fill_(7), a.sm.fill_(7), a.conf.fill_(0.125)
    a.table.copy_(a.i32(pages))
    ref = a.i32(np.ones(n_pages))
    a.layer, a.map = lg.paged_layer(k, v, 4), lg.page_map(a.table, a.pos, a.len, ref, ps)
    a.call()
    for x, y in zip(small, a.results()):
        np.testing.assert_array_equal(x, y)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), float("-inf")])
def test_values_in_slots_that_are_not_seen(dtype, value):
    """Rows of no live slot, rows of later tokens of the chunk, and rows that the window hides hold infinities and
    NaN: only tokens that see them change."""
    clean = Attend(dtype, 128, 6, 2, 16, [90, 40, 0], [30, 1, 3], window=25, sinks=4, seed=11, holes=False, cap_pages=12)
    a = Attend(dtype, 128, 6, 2, 16, [90, 40, 0], [30, 1, 3], window=25, sinks=4, seed=11, holes=False, cap_pages=12)
    live = np.zeros((len(a.k), a.ps), bool)
    for b, n in enumerate(a.n):
        for j in range(a.have[b] + n):
            live[a.table_h[b, j // a.ps], j % a.ps] = True
    dead = torch.as_tensor(~live, device="cuda")[:, None, :, None]
    for x in (a.k, a.v):
        x.masked_fill_(dead, value)
    # sequence 0: slot 30 (behind the sinks, out of every window), slot 110 (token 20: seen by tokens 20 .. 29);
    # sequence 1: slot 10 (out of the window); sequence 2: slot 2 (its last token)
    for b, j in ((0, 30), (0, 110), (1, 10), (2, 2)):
        p = int(a.table_h[b, j // a.ps])
        a.v[p, :, j % a.ps, 5] = value
        a.k[p, :, j % a.ps, 9] = value
    clean.call()
    a.call()
    want, got = clean.results(), a.results()
    hit = np.zeros(a.T, bool)
    hit[20:30] = True
    hit[33] = True
    # A tile with such a value is multiplied term by term in float32. Against the matrix product that is, in
    # bfloat16, the rounding of each weight and both outputs' rounding, 3 x 2^-8 max |v|; in float32 the
    # order of at most 130 terms, twice.
    most = float(clean.v.abs().max())
    far = 3 * 2.0 ** -8 * most if dtype is BF else 2 * 130 * 2.0 ** -24 * most
    for x, y in zip(want[:3], got[:3]):
        ok = ~hit
        if x.ndim == 3:
            assert np.isfinite(y[ok]).all()
            np.testing.assert_allclose(y[ok], x[ok], rtol=0, atol=far)
        else:
            np.testing.assert_array_equal(x[ok], y[ok])
    clean_rows = Attend(dtype, 128, 6, 2, 16, [90, 40, 0], [30, 1, 3], window=25, sinks=4, seed=11, holes=False, cap_pages=12)
    clean_rows.check([np.where(hit.reshape([-1] + [1] * (x.ndim - 1)), x, y) if len(x) == a.T else x
                      for x, y in zip(want, got)])


@pytest.mark.parametrize("dtype", [BF, F32])
def test_infinite_values_are_seen(dtype):
    """A slot that a token sees and whose V is infinite gives it that infinity; the other values are as ever."""
    a = Attend(dtype, 64, 4, 2, 16, [40], [2], seed=12, holes=False, gain=0.5)
    p, row = int(a.table_h[0, 41 // 16]), 41 % 16  # the last token's own slot: token 0 does not see it
    a.v[p, :, row, 3] = float("inf")
    a.v[p, :, row, 4] = float("-inf")
    a.call()
    out = a.results()[0]
    assert (out[1, :, 3] == np.inf).all() and (out[1, :, 4] == -np.inf).all()
    assert np.isfinite(out[0]).all() and np.isfinite(np.delete(out[1], [3, 4], 1)).all()


@pytest.mark.parametrize("dtype, D, hq, hkv", [(BF, 128, 8, 2), (BF, 64, 6, 6), (F32, 128, 4, 1), (F32, 64, 4, 4)])
@pytest.mark.parametrize("chunk", [1, 3, 70])
@pytest.mark.parametrize("window, sinks", [(100, 4), (2500, 40), (9000, 0), (30000, 600)])
def test_windows_over_pruned_history(dtype, D, hq, hkv, chunk, window, sinks):
    """Histories thinned out eight to one, and a few slots behind one long gap: a window holds far fewer slots
    than positions."""
    a = Attend(dtype, D, hq, hkv, 32, [3200, 1500, 40], [1, chunk, chunk], window=window, sinks=sinks, seed=window + chunk)
    a.pos_h = np.cumsum(np.where(np.arange(a.pos_h.shape[1]) < 30, 1, a.r.randint(1, 16, a.pos_h.shape)), 1) - 1
    a.pos_h[1, 1450:] += 20000
    a.alloc()
    a.call()
    a.check()


@pytest.mark.parametrize("dtype", [BF, F32])
def test_infinite_value_of_a_vanishing_weight(dtype):
    """Waves that see a tile whole and waves that do not share it: a slot whose weight rounds to 0 and whose V is
    infinite gives every token that sees it that infinity, whichever wave comes to the tile first."""
    a = Attend(dtype, 64, 1, 1, 16, [0], [128], seed=14, holes=False)
    a.q.fill_(1.0)
    a.k.zero_()
    p = int(a.table_h[0, 0])
    a.k[p, 0, 10] = -1000.0  # a score of -8000
    a.v[p, 0, 10, 3] = float("inf")
    for _ in range(8):
        a.call()
        out = a.results()[0][:128, 0]
        assert np.isfinite(out[:10]).all() and (out[10:, 3] == np.inf).all()
        assert np.isfinite(np.delete(out, 3, 1)).all()


def test_large_scores():
    """Scores of several hundred: weights of the far ones are 0, the lse is the largest score."""
    a = Attend(BF, 128, 4, 2, 16, [300, 20], [3, 40], seed=13, gain=60.0)
    a.call()
    a.check()
    a = Attend(F32, 64, 4, 2, 16, [300], [3], seed=13, gain=200.0)
    a.call()
    a.check()


@pytest.mark.parametrize("dtype", [BF, F32])
def test_missing_pages(dtype):
    """Slots whose column names no page of the pool are not seen; a token with none left gets an empty row."""
    a = Attend(dtype, 64, 4, 2, 16, [70, 10, 33], [4, 2, 1], seed=14)
    a.table_h[0, 1], a.table_h[0, 3] = -1, 10 ** 9
    a.table_h[1, 0] = -5
    a.table_h[2, :] = len(a.k)
    a.see = {0: ~np.isin(np.arange(a.P * 16) // 16, [1, 3]), 1: np.zeros(a.P * 16, bool), 2: np.zeros(a.P * 16, bool)}
    for b in a.see:
        a.see[b] = a.see[b][:a.have[b] + a.n[b]]
    a.alloc()
    a.call()
    a.check()


def test_refused_sequences():
    """base < 0, a chunk longer than max_chunk, a base that leaves no room: rows untouched, conf NaN; an empty one
    keeps its conf."""
    a = Attend(BF, 64, 8, 2, 16, [20, 30, 40, 5, 6], [3, 4, 30, 0, 2], seed=15)
    a.base_h = np.array([20, -1, 40, -1, 10 ** 6])
    a.chunk = 29
    a.skip = {1, 2, 4}
    a.alloc()
    a.call()
    a.check()


def test_without_statistics():
    a = Attend(BF, 128, 4, 2, 16, [40, 700], [3, 1], seed=16)
    a.call(statistics=False)
    a.check(statistics=False)


@pytest.mark.parametrize("suffix", [[0, 0], [2 ** 31 - 1, 2 ** 31 - 1], [1, 1], [33, 50]])
def test_suffix_widths(suffix):
    for dtype in (BF, F32):
        a = Attend(dtype, 64, 4, 2, 16, [40, 100], [70, 1], seed=17, suffix=suffix)
        a.call()
        a.check()


def test_extreme_positions():
    """Positions up to 2^30 and widths that would pass the least integer."""
    a = Attend(BF, 64, 4, 2, 16, [40], [3], seed=18, window=2 ** 31 - 1, sinks=2 ** 31 - 1, suffix=[2 ** 31 - 1])
    a.pos_h = a.pos_h + 2 ** 30 - 400
    a.alloc()
    a.call()
    a.check()


@pytest.mark.parametrize("B", [65, 130])
def test_many_sequences(B):
    n = [(b * 5) % 4 if b % 9 else 20 for b in range(B)]
    a = Attend(BF, 64, 4, 2, 16, [(b * 13) % 50 for b in range(B)], n, seed=19)
    a.call()
    a.check()


def test_deterministic_and_on_another_stream():
    a = Attend(BF, 128, 28, 4, 16, [500, 30, 1200], [1, 60, 1], seed=20, window=400, sinks=4)
    a.call()
    want = a.results()
    for _ in range(3):
        for x in (a.out, a.lse, a.sm):
            x.fill_(7.0)
        a.conf.fill_(0.125)
        a.ws.fill_(0xff)
        st = torch.cuda.Stream()
        st.wait_stream(torch.cuda.current_stream())
        a.call(stream=st)
        st.synchronize()
        for x, y in zip(want, a.results()):
            np.testing.assert_array_equal(x, y)


def test_conf_keeps_the_larger_and_nan():
    a = Attend(BF, 64, 4, 2, 16, [40, 40], [1, 1], seed=21)
    a.conf.copy_(torch.tensor([0.9999, float("nan")]))
    a.call()
    conf = a.results()[3]
    assert conf[0] >= np.float32(0.9999) and np.isnan(conf[1])


def test_binding_refuses():
    from paper_2604_10044_amd import lg
    a = Attend(BF, 64, 4, 2, 16, [40], [3], seed=22)
    for name, bad in (("q", a.q.float()), ("out", a.out[:-1]), ("lse", a.lse.double()), ("sm", a.sm[:-1]),
                      ("conf", a.conf.cpu()), ("base", a.base.long()), ("q_start", a.q_start[:-1]),
                      ("out", a.out.transpose(0, 1)), ("ws", a.ws[:0].clone())):
        was = getattr(a, name)
        setattr(a, name, bad)
        with pytest.raises(lg.LGError):
            a.call()
        setattr(a, name, was)
    a.call()
    a.check()
