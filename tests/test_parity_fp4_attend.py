"""lg_paged_attend_fp4 against attention in 64 bits (oracle/paged.py) on the values that the 4-bit pages stand for, at
the sizes, masks and values where it can go wrong.

The error bounds are those of tests/test_parity_paged_attend.py, where they are derived from the count of roundings: keys
and values are exact as bfloat16, the products of float32 calls are sums of exact ones (three bfloat16 terms hold all 24
bits), and a bfloat16 call's weights are rounded by at most 2^-8. Steps of few rows have their own bound in
test_weights_of_few_rows. One term more: values in 4 bits are often 0 exactly, and an output may then be the sum of vanishing
weights alone. A weight below 2^-126 of the row's largest is no normal float32 and may become 0, as may the last terms of one
that is not far above it (each below 2^-126 too): of n slots and at most three terms, n 2^-124 max |v| together."""
import numpy as np
import pytest
import torch

from oracle import fp4, paged
from test_parity_paged_attend import BF, F32, SMALL, Attend

pytestmark = pytest.mark.gpu


class Attend4(Attend):
    """The same step over 4-bit pages: k and v hold the values that the pages stand for."""

    def alloc(self):
        lg, dev = self.lg, "cuda"
        self.bytes = []
        for x in (self.k, self.v):
            b = fp4.pages(x.double().cpu().numpy())
            x.copy_(torch.as_tensor(fp4.values(*fp4.unpack(b, self.ps, self.D))).to(x.dtype))
            self.bytes.append(torch.as_tensor(b, device=dev))
        self.table, self.pos = self.i32(self.table_h), self.i32(self.pos_h)
        self.base, self.q_start, self.sw = self.i32(self.base_h), self.i32(self.start_h), self.i32(self.sw_h)
        self.len, self.ref = self.i32(self.base_h), self.i32(np.ones(len(self.k)))
        self.layer = lg.paged_layer_fp4(*self.bytes, self.hq, self.ps, self.D)
        self.map = lg.page_map(self.table, self.pos, self.len, self.ref, self.ps)
        self.out = torch.full_like(self.q, 7.0)
        self.lse = torch.full((self.T, self.hq), 7.0, device=dev)
        self.sm = torch.full((self.T, self.hq), 7.0, device=dev)
        self.conf = torch.full((len(self.n),), 0.125, device=dev)
        size = lg.lg_paged_attend_fp4_workspace(self.layer, self.map, self.dtype, self.T, self.chunk)
        self.ws = torch.full((size,), 0xff, dtype=torch.uint8, device=dev)  # NaN: nothing is read unwritten

    def call(self, stream=None, statistics=True):
        self.lg.lg_paged_attend_fp4(self.layer, self.map, self.q, self.out, self.q_start, self.base, self.chunk, self.window, self.sinks,
                                    self.sw if statistics else None, self.lse, self.sm if statistics else None,
                                    self.conf if statistics else None, self.ws, stream=stream)

    def check(self, got=None, statistics=True, tokens=None):
        out, lse, sm, conf = self.results() if got is None else got
        G, D, ps = self.hq // self.hkv, self.D, self.ps
        k, v, q = (x.double().cpu().numpy() for x in (self.k, self.v, self.q))
        half, w = (2.0 ** -8, 2.0 ** -8) if self.dtype is BF else (2.0 ** -24, 0.0)
        for b, n in enumerate(self.n):
            rows = np.arange(self.start_h[b], self.start_h[b] + n)
            if b in self.skip:
                assert (out[rows] == 7).all() and (lse[rows] == 7).all() and (sm[rows] == 7).all()
                assert n == 0 or not statistics or np.isnan(conf[b])
                continue
            slots = np.arange(self.have[b] + n)
            page = self.table_h[b, slots // ps]
            page = np.where((page >= 0) & (page < len(k)), page, 0)
            pos, see = self.pos_h[b, :len(slots)], self.see.get(b)
            best = 0.125
            for i in np.arange(n) if tokens is None or n == 0 else np.unique(np.clip(tokens, -n, n - 1) % n):
                e, row = self.have[b] + i + 1, rows[i]
                for h in range(self.hkv):
                    kk, vv = (x[page[:e], h, slots[:e] % ps] for x in (k, v))
                    o, ls, ms, av, big = (x[0] for x in paged.attend(
                        q[row, h * G:(h + 1) * G][None], kk, vv, pos[:e], e - 1, self.window, self.sinks, int(self.sw_h[b]),
                        None if see is None else see[:e]))
                    heads, what = slice(h * G, (h + 1) * G), (b, h, i)
                    err = ((D + 8) * big + 4 * e / 32 + 144) * 2.0 ** -24
                    tol = ((2 * err[:, None] + w) * av) * (1 + half) + half * np.abs(o) + e * 2.0 ** -124 * np.abs(vv).max()
                    assert (np.abs(out[row, heads] - o) <= tol).all(), (what, np.abs(out[row, heads] - o).max())
                    some = np.isfinite(ls)
                    assert (lse[row, heads][~some] == -np.inf).all() and (out[row, heads][~some] == 0).all(), what
                    assert (np.abs(lse[row, heads] - ls)[some] <= (err + 2.0 ** -22 * (np.abs(ls) + big))[some]).all(), what
                    if statistics:
                        assert (np.abs(sm[row, heads] - ms) <= 2 * err * ms + e * 2.0 ** -126).all(), what
                if i == n - 1:
                    best = max(best, sm[row].max())
            if statistics and (n == 0 or tokens is None or n - 1 in np.clip(tokens, -n, n - 1) % n):
                assert conf[b] == best, (b, conf[b], best)
        behind = self.start_h[-1]
        assert (out[behind:] == 7).all() and (lse[behind:] == 7).all() and (sm[behind:] == 7).all()
        if not statistics:
            assert (sm == 7).all() and (conf == 0.125).all()

    def exponents(self, x):
        """The exponent bytes of the pages, [n_pages][Hkv][page_size][D / 32], as a view."""
        return self.bytes[x][..., self.ps * self.D // 2:].unflatten(-1, (self.ps, self.D // 32))


MORE = [
    (F32, 128, 28, 4, 64, [0, 1, 63, 64, 65, 200], [1, 1, 1, 1, 1, 1]),
    (F32, 128, 6, 2, 256, [250, 10], [70, 1]),
    (BF, 64, 3, 3, 16, [7, 0], [16, 17]),
    (BF, 64, 8, 2, 16, [90, 14, 0], [5, 4, 8]),   # 20, 16 and 32 rows
]


@pytest.mark.parametrize("window,sinks", [(0, 0), (1, 0), (7, 4), (40, 20), (100000, 4)])
@pytest.mark.parametrize("dtype,D,hq,hkv,ps,have,n", SMALL + MORE)
def test_small(dtype, D, hq, hkv, ps, have, n, window, sinks):
    a = Attend4(dtype, D, hq, hkv, ps, have, n, window=window, sinks=sinks, seed=D + hq + window)
    a.call()
    a.check()


@pytest.mark.parametrize("dtype,D,hq,hkv,ps,have,n,window,sinks", [
    (BF, 128, 12, 2, 16, [5000, 333], [1, 1], 0, 0),          # few rows: many splits, joined
    (BF, 128, 12, 2, 64, [9000], [1], 512, 32),               # the window skips most of the cache
    (BF, 64, 4, 4, 16, [4000], [64], 0, 0),                   # many rows, split
    (BF, 128, 28, 4, 64, [2000, 100, 1500], [1, 150, 20], 700, 32),
    (F32, 128, 8, 2, 16, [3000], [1], 0, 0),
    (F32, 64, 4, 1, 32, [1500, 0], [40, 300], 600, 4),
    (F32, 128, 8, 2, 16, [2000, 31], [50, 1], 0, 0),
])
def test_long(dtype, D, hq, hkv, ps, have, n, window, sinks):
    a = Attend4(dtype, D, hq, hkv, ps, have, n, window=window, sinks=sinks, seed=7)
    a.call()
    a.check(tokens=np.array([0, 1, 17, 63, 64, -1]))


@pytest.mark.parametrize("dtype,D,hq,hkv,batch", [
    (BF, 128, 4, 4, 32), (BF, 128, 14, 2, 45), (BF, 128, 8, 1, 70), (F32, 128, 4, 2, 50), (BF, 64, 16, 4, 32), (BF, 128, 8, 8, 40),
    (F32, 64, 16, 1, 130),
    (BF, 128, 8, 4, 50),      # 200 pairs: 16 waves a workgroup
    (BF, 64, 12, 4, 40),
    (F32, 128, 8, 4, 50),
    (BF, 128, 40, 40, 3),     # one query head a KV head
])
def test_decode_batches(dtype, D, hq, hkv, batch):
    """A token a sequence at batch sizes that take each launch of the decode step."""
    have = [(37 * b) % 700 for b in range(batch)]
    for window, sinks in ((0, 0), (100, 5)):
        a = Attend4(dtype, D, hq, hkv, 16, have, [1] * batch, window=window, sinks=sinks, seed=batch)
        a.call()
        a.check()


@pytest.mark.parametrize("dtype,D,hq,hkv,have,n", [
    (BF, 128, 8, 2, [950, 3, 500], [1, 1, 1]), (BF, 128, 4, 1, [700], [8]), (BF, 128, 8, 4, [1400] + [60] * 15, [1] * 16),
    (F32, 128, 8, 2, [950, 3, 500], [1, 4, 4]), (F32, 128, 8, 2, [950, 3, 500], [5, 1, 0]), (F32, 64, 16, 4, [300, 33], [8, 1]),
    (F32, 64, 5, 1, [40, 0], [6, 3]), (F32, 128, 2, 1, [130] * 70, [16] + [9] * 69), (BF, 128, 3, 3, [90] * 40, [16] + [1] * 39),
    (BF, 64, 2, 1, [130] * 70, [16] + [9] * 69),
])
def test_few_rows(dtype, D, hq, hkv, have, n):
    """Steps without long chunks at the edges of their launches."""
    a = Attend4(dtype, D, hq, hkv, 16, have, n, seed=sum(n) + D)
    a.call()
    a.check(tokens=np.array([0, 1, 3, 4, -1]))


@pytest.mark.parametrize("dtype,D,hq,hkv,have,n", [
    (BF, 128, 8, 2, [2900] + [60] * 39, [1] * 40),   # 80 pairs of long capacity: splits, two workgroups a CU
    (BF, 128, 14, 2, [2900] + [60] * 39, [4] + [1] * 39),  # of 28 rows: one a CU
    (BF, 64, 8, 2, [1900] + [60] * 39, [1] * 40),
    (F32, 128, 8, 2, [1500] + [60] * 39, [1] * 40),
    (F32, 64, 8, 2, [1900] + [60] * 39, [2] * 40),
    (BF, 128, 8, 8, [9000], [1]),                    # 32 splits, and 64
    (BF, 64, 4, 1, [17000], [2]),
    (F32, 128, 4, 1, [17000], [1]),
])
def test_splits(dtype, D, hq, hkv, have, n):
    a = Attend4(dtype, D, hq, hkv, 32, have, n, seed=sum(n) + D)
    a.call()
    a.check()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("n", [1, 6, 50])
def test_nan_in_one_of_several_splits(dtype, n):
    """Keys and values that stand for NaN in a slot that one split of several has."""
    for which in (0, 1):
        a = Attend4(dtype, 128, 8, 2, 16, [3000, 70], [n, 1], seed=26, holes=False)
        a.call()
        want = a.results()
        assert np.isfinite(want[0][:n + 1]).all()
        p = int(a.table_h[0, 1234 // 16])
        a.exponents(which)[p, 1, 1234 % 16, 3] = 255
        a.call()
        got = a.results()
        rows, heads = slice(0, n), slice(4, 8)
        if which == 0:
            assert np.isnan(got[0][rows, heads]).all() and np.isnan(got[1][rows, heads]).all() and np.isnan(got[3][0])
            for x, y in zip(got[:3], want[:3]):
                x[rows, heads] = y[rows, heads]
            got[3][0] = want[3][0]
        else:
            assert np.isnan(got[0][rows, heads, 96:]).all()
            got[0][rows, heads, 96:] = want[0][rows, heads, 96:]
        for x, y in zip(got, want):
            np.testing.assert_array_equal(x, y)


@pytest.mark.parametrize("dtype,D,hq,hkv,n", [(BF, 128, 8, 2, [1, 4, 8]), (BF, 64, 16, 1, [1, 2, 2]), (BF, 128, 4, 4, [16, 20, 32])])
def test_weights_of_few_rows(dtype, D, hq, hkv, n):
    """A sequence's weights are within 2^-16 where it has at most 32 rows: outputs that nearly cancel keep their digits."""
    a = Attend4(dtype, D, hq, hkv, 16, [300, 77, 1000], n, seed=5, holes=False)
    for b in range(3):  # every odd slot's values are the negatives of the slot's before it, and the keys are alike
        for c in range(a.P):
            p = int(a.table_h[b, c])
            a.v[p, :, 1::2] = -a.v[p, :, 0::2]
            a.k[p, :, 1::2] = a.k[p, :, 0::2]
    a.alloc()
    a.call()
    out = a.results()[0]
    k, v, q = (x.double().cpu().numpy() for x in (a.k, a.v, a.q))
    G = hq // hkv
    for b in range(3):
        m = a.have[b] + n[b]
        page, off = a.table_h[b, np.arange(m) // 16], np.arange(m) % 16
        for h in range(hkv):
            rows = np.arange(a.start_h[b], a.start_h[b] + n[b])
            o, _, _, av, big = paged.attend(q[rows][:, h * G:(h + 1) * G], k[page, h, off], v[page, h, off], np.arange(m), a.have[b], 0, 0, 1)
            err = ((D + 8) * big + 4 * m / 32 + 144) * 2.0 ** -24
            tol = (2 * err[..., None] + 2.0 ** -16) * av * (1 + 2.0 ** -8) + 2.0 ** -8 * np.abs(o)
            assert (np.abs(out[rows][:, h * G:(h + 1) * G] - o) <= tol).all(), (b, h)


def test_long_capacity():
    """More slots of capacity than a split may have: most splits are empty."""
    a = Attend4(BF, 64, 32, 32, 256, [3, 700, 40, 0, 90, 2000, 31, 64, 5], [1, 1, 2, 1, 0, 1, 1, 40, 1], seed=23)
    more = 600 - a.P
    a.table_h = np.concatenate([a.table_h, np.full((9, more), -1)], 1)
    a.pos_h = np.concatenate([a.pos_h, np.full((9, more * 256), -1)], 1)
    a.alloc()
    a.call()
    a.check(tokens=np.array([0, 1, 39]))


@pytest.mark.parametrize("dtype", [BF, F32])
def test_long_prompt(dtype):
    """Thousands of tokens in one chunk behind others, two sequences."""
    a = Attend4(dtype, 128, 8, 2, 64, [1000, 3], [2100, 700], seed=8, holes=False)
    a.call()
    a.check(tokens=np.array([0, 1, 31, 32, 500, 1023, 1024, 2047, -2, -1]))


def test_large_offsets():
    """Pages whose bytes lie beyond 2^32."""
    from paper_2604_10044_amd import lg
    n_pages, ps, hkv, D = 300000, 128, 2, 128  # 5.2 GB each of K and V
    k = torch.zeros(n_pages, hkv, lg.fp4_page_bytes(ps, D), dtype=torch.uint8, device="cuda")
    v = torch.zeros_like(k)
    for n in ([3, 20], [1, 3]):
        a = Attend4(BF, D, 4, hkv, ps, [200, 100], n, seed=9)
        pages = np.array([[299999, 5, 265535], [265536, 290000, 1]])[:, :a.P]
        for b in range(2):
            for c in range(a.P):
                k[int(pages[b, c])], v[int(pages[b, c])] = (x[int(a.table_h[b, c])] for x in a.bytes)
        a.call()
        small = a.results()
        a.check(small)
        a.out.fill_(7), a.lse.fill_(7), a.sm.fill_(7), a.conf.fill_(0.125)
        a.table.copy_(a.i32(pages))
        a.layer, a.map = lg.paged_layer_fp4(k, v, 4, ps, D), lg.page_map(a.table, a.pos, a.len, a.i32(np.ones(n_pages)), ps)
        a.call()
        for x, y in zip(small, a.results()):
            np.testing.assert_array_equal(x, y)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("chunks", [[30, 1, 3], [4, 1, 3]])
def test_slots_that_are_not_seen(dtype, chunks):
    """Rows of no live slot hold any bytes, and rows of later tokens of the chunk and rows that the window hides stand for
    NaN: tokens that do not see them keep their results bit for bit, those that do get NaN where the definition says."""
    def make():
        return Attend4(dtype, 128, 6, 2, 16, [90, 40, 0], chunks, window=25, sinks=4, seed=11, holes=False, cap_pages=12)

    clean, a = make(), make()
    live = np.zeros((len(a.k), a.ps), bool)
    for b, n in enumerate(a.n):
        for j in range(a.have[b] + n):
            live[a.table_h[b, j // a.ps], j % a.ps] = True
    dead = torch.as_tensor(~live, device="cuda")[:, None, :, None].expand(-1, 2, -1, 4)
    g = torch.Generator(device="cuda").manual_seed(1)
    for x in range(2):
        e = a.exponents(x)
        e[dead] = torch.randint(0, 256, (int(dead.sum()),), generator=g, device="cuda", dtype=torch.uint8)
    # sequence 0: slot 30 (behind the sinks, out of every window), the last token's slot; sequence 1: slot 10 (out of
    # the window), slot 39 (seen: values alone); sequence 2: slot 2 (its last token: keys alone)
    last = 90 + chunks[0] - 1
    for b, j, ks, vs in ((0, 30, 255, 254), (0, last, 0, 253), (1, 10, 255, 255), (1, 39, 0, 255), (2, 2, 255, 0)):
        p = int(a.table_h[b, j // a.ps])
        if ks:
            a.exponents(0)[p, :, j % a.ps, 1] = ks
        if vs:
            a.exponents(1)[p, :, j % a.ps, 2] = vs
    clean.call()
    a.call()
    want, got = clean.results(), a.results()
    starts = a.start_h
    values_hit, keys_hit = np.zeros(a.T, bool), np.zeros(a.T, bool)
    values_hit[[starts[1] - 1, starts[1]]] = True
    keys_hit[starts[3] - 1] = True
    for i, (x, y) in enumerate(zip(want[:3], got[:3])):
        x, y = x.copy(), y.copy()
        if i == 0:
            assert np.isnan(y[values_hit][..., 64:96]).all() and np.isnan(y[keys_hit]).all()
            y[values_hit, :, 64:96] = x[values_hit, :, 64:96]
        else:
            assert np.isnan(y[keys_hit]).all()
        np.testing.assert_array_equal(x[~keys_hit], y[~keys_hit])
    np.testing.assert_array_equal(want[3][:2], got[3][:2])
    assert np.isnan(got[3][2])


@pytest.mark.parametrize("dtype", [BF, F32])
def test_nan_of_a_vanishing_weight(dtype):
    """A slot whose weight rounds to 0 and whose values stand for NaN gives it to every token that sees it, in its 32
    values alone, whichever wave comes to the tile first; in a chunk and in a decode step."""
    for hkv, n in ((1, 128), (1, 20), (2, 1)):
        a = Attend4(dtype, 64, hkv, hkv, 16, [0 if n > 1 else 50], [n], seed=14, holes=False)
        a.q.fill_(1.0)
        a.k.zero_()
        p = int(a.table_h[0, 0])
        a.k[p, :, 10] = -1000.0  # a score below -6000
        a.alloc()
        a.exponents(1)[p, :, 10, 1] = 255
        for _ in range(4):
            a.call()
            out = a.results()[0][:n]
            assert np.isfinite(out[:10 if n > 1 else 0]).all() and np.isnan(out[10 if n > 1 else 0:, :, 32:]).all()
            assert np.isfinite(out[..., :32]).all()


@pytest.mark.parametrize("dtype", [BF, F32])
def test_nan_without_any_weight(dtype):
    """Queries of infinity before keys below 0: every score is -inf and no slot has weight. 0, but NaN in the 32 values of a
    group that stands for it; in a chunk, in a step of one workgroup and in one of several splits."""
    for hkv, have, n in ((1, 0, 128), (2, 50, 1), (2, 3000, 1), (2, 3000, 40)):
        a = Attend4(dtype, 64, hkv, hkv, 16, [have], [n], seed=26, holes=False)
        a.q.fill_(float("inf"))
        a.k.fill_(-1.0)
        a.alloc()
        a.exponents(1)[int(a.table_h[0, 0]), :, 10, 1] = 255
        a.call()
        out, lse, sm, _ = a.results()
        first = max(0, 10 - have)  # the first token that sees slot 10
        assert (lse[:n] == -np.inf).all() and (sm[:n] == 0).all()
        assert (out[:n, :, :32] == 0).all() and (out[:first] == 0).all() and np.isnan(out[first:n, :, 32:]).all()


@pytest.mark.parametrize("dtype, D, hq, hkv", [(BF, 128, 8, 2), (BF, 64, 6, 6), (F32, 128, 4, 1), (F32, 64, 4, 4)])
@pytest.mark.parametrize("chunk", [1, 3, 70])
@pytest.mark.parametrize("window, sinks", [(100, 4), (2500, 40), (9000, 0), (30000, 600)])
def test_windows_over_pruned_history(dtype, D, hq, hkv, chunk, window, sinks):
    """Histories thinned out eight to one, and a few slots behind one long gap."""
    a = Attend4(dtype, D, hq, hkv, 32, [3200, 1500, 40], [1, chunk, chunk], window=window, sinks=sinks, seed=window + chunk)
    a.pos_h = np.cumsum(np.where(np.arange(a.pos_h.shape[1]) < 30, 1, a.r.randint(1, 16, a.pos_h.shape)), 1) - 1
    a.pos_h[1, 1450:] += 20000
    a.alloc()
    a.call()
    a.check(tokens=np.array([0, 1, 2, 31, 63, -1]))


def test_large_scores():
    """Scores of several hundred: weights of the far ones are 0, the lse is the largest score."""
    for dtype, D, gain, n in ((BF, 128, 60.0, [3, 40]), (F32, 64, 200.0, [3, 33])):
        a = Attend4(dtype, D, 4, 2, 16, [300, 20], n, seed=13, gain=gain)
        a.call()
        a.check()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("n", [[4, 2, 1], [40, 33, 1]])
def test_missing_pages(dtype, n):
    """Slots whose column names no page of the pool are not seen; a token with none left gets an empty row."""
    a = Attend4(dtype, 64, 4, 2, 16, [70, 10, 33], n, seed=14)
    a.table_h[0, 1], a.table_h[0, 3] = -1, 10 ** 9
    a.table_h[1, :] = -5
    a.table_h[2, :] = len(a.k)
    a.see = {0: ~np.isin(np.arange(a.P * 16) // 16, [1, 3]), 1: np.zeros(a.P * 16, bool), 2: np.zeros(a.P * 16, bool)}
    for b in a.see:
        a.see[b] = a.see[b][:a.have[b] + a.n[b]]
    a.alloc()
    a.call()
    a.check()


def test_refused_sequences():
    """base < 0, a chunk longer than max_chunk, a base that leaves no room: rows untouched, conf NaN."""
    for dtype in (BF, F32):
        a = Attend4(dtype, 64, 8, 2, 16, [20, 30, 40, 5, 6], [3, 4, 30, 0, 2], seed=15)
        a.base_h = np.array([20, -1, 40, -1, 10 ** 6])
        a.chunk = 29
        a.skip = {1, 2, 4}
        a.alloc()
        a.call()
        a.check()


@pytest.mark.parametrize("dtype", [BF, F32])
def test_max_chunk_is_a_bound(dtype):
    """A larger max_chunk than any sequence brings, with the launch that belongs to it."""
    for chunk in (1, 8, 33, 4000):
        a = Attend4(dtype, 128, 4, 1, 16, [100, 900, 0], [1, 1, 1], seed=16)
        a.chunk = chunk
        a.alloc()
        a.call()
        a.check()


def test_without_statistics():
    for n in ([3, 1], [60, 1]):
        a = Attend4(BF, 128, 4, 2, 16, [40, 700], n, seed=16)
        a.call(statistics=False)
        a.check(statistics=False)


@pytest.mark.parametrize("suffix", [[0, 0], [2 ** 31 - 1, 2 ** 31 - 1], [1, 1], [33, 50]])
def test_suffix_widths(suffix):
    for dtype in (BF, F32):
        a = Attend4(dtype, 64, 4, 2, 16, [40, 100], [70, 1], seed=17, suffix=suffix)
        a.call()
        a.check()


def test_extreme_positions():
    """Positions up to 2^30 and widths that would pass the least integer."""
    a = Attend4(BF, 64, 4, 2, 16, [40], [3], seed=18, window=2 ** 31 - 1, sinks=2 ** 31 - 1, suffix=[2 ** 31 - 1])
    a.pos_h = a.pos_h + 2 ** 30 - 400
    a.alloc()
    a.call()
    a.check()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("B", [65, 130])
def test_many_sequences(B, dtype):
    n = [(b * 5) % 4 if b % 9 else 20 for b in range(B)]
    a = Attend4(dtype, 64, 4, 2, 16, [(b * 13) % 50 for b in range(B)], n, seed=19)
    a.call()
    a.check()


@pytest.mark.parametrize("dtype", [BF, F32])
def test_splits_of_a_sequence_behind_empty_ones(dtype):
    """A workgroup that joins splits has rows of two sequences, with many of no rows, or a few, between them."""
    for empty in (1, 2, 3, 7, 60):
        n = [3] + [0] * empty + [2, 0, 1]
        a = Attend4(dtype, 64, 1, 1, 16, [2000] + [5] * empty + [1900, 3, 2000], n, seed=27)
        a.call()
        a.check()


@pytest.mark.parametrize("dtype", [BF, F32])
def test_rows_before_the_first_sequence(dtype):
    """q_start need not begin at 0."""
    for n in ([3, 1], [40, 2]):
        a = Attend4(dtype, 64, 4, 2, 16, [40, 7], n, seed=24, extra=6)
        a.start_h = a.start_h + 4
        a.alloc()
        a.call()
        got = a.results()
        assert (got[0][:4] == 7).all() and (got[1][:4] == 7).all() and (got[2][:4] == 7).all()
        a.check(got)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_deterministic_and_on_another_stream(dtype):
    for n in ([1, 60, 1], [1, 1, 4]):
        a = Attend4(dtype, 128, 28, 4, 16, [500, 30, 1200], n, seed=20, window=400, sinks=4)
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
    a = Attend4(BF, 64, 4, 2, 16, [40, 40], [1, 1], seed=21)
    a.conf.copy_(torch.tensor([0.9999, float("nan")]))
    a.call()
    conf = a.results()[3]
    assert conf[0] >= np.float32(0.9999) and np.isnan(conf[1])


def test_queries_that_are_not_finite():
    """A query with an infinity or NaN spoils its own row alone."""
    for dtype in (BF, F32):
        for n in ([3], [40]):
            a = Attend4(dtype, 64, 4, 2, 16, [40], n, seed=25)
            a.call()
            want = a.results()[0].copy()
            a.q[1, 2, 5], a.q[2, 0, 7] = float("nan"), float("inf")
            a.call()
            got = a.results()[0]
            assert np.isnan(got[1, 2]).all()
            got[1, 2], got[2, 0] = want[1, 2], want[2, 0]
            np.testing.assert_array_equal(got, want)


def test_binding_refuses():
    from paper_2604_10044_amd import lg
    a = Attend4(BF, 64, 4, 2, 16, [40], [3], seed=22)
    for name, bad in (("q", a.q.float()), ("q", a.q.half()), ("out", a.out[:-1]), ("lse", a.lse.double()), ("sm", a.sm[:-1]),
                      ("conf", a.conf.cpu()), ("base", a.base.long()), ("q_start", a.q_start[:-1]), ("out", a.out.transpose(0, 1)),
                      ("ws", a.ws[:0].clone())):
        was = getattr(a, name)
        setattr(a, name, bad)
        with pytest.raises(lg.LGError):
            a.call()
        setattr(a, name, was)
    with pytest.raises(lg.LGError):
        lg.lg_paged_attend(a.layer, a.map, a.q, a.out, a.q_start, a.base, 3, 0, 0, None, a.lse, None, None, a.ws)
    a.call()
    a.check()


@pytest.mark.parametrize("dtype,D,n", [(BF, 128, [1, 4]), (BF, 64, [1, 1]), (BF, 128, [40, 1]), (BF, 64, [70, 2]), (F32, 128, [2, 1]),
                                       (F32, 64, [1, 3]), (F32, 128, [40, 1]), (F32, 64, [1, 50])])
@pytest.mark.parametrize("keys,values", [((0, 1, 2), ()), ((248, 250, 252), ()), ((), (0, 1, 2)), ((), (236, 238, 240)), ((0, 1), (0, 2))])
def test_exponents_at_the_ends(dtype, D, n, keys, values):
    """Groups with the least and the largest units, and queries that bring the scores to ordinary size. Queries are bfloat16
    numbers. Products and sums of values below 2^-126 are off by half a step of the least numbers, 2^-149 in float32: three
    terms of e slots, their sums and the scaling; a bfloat16 result by half of 2^-133."""
    a = Attend4(dtype, D, 4, 2, 16, [70, 10], n, seed=31, holes=False)
    for which, units in ((0, keys), (1, values)):
        if units:
            e = a.exponents(which)
            e.copy_(torch.as_tensor(a.r.choice(units, tuple(e.shape)).astype(np.uint8), device="cuda"))
            x = (a.k, a.v)[which]
            x.copy_(torch.as_tensor(fp4.values(*fp4.unpack(a.bytes[which].cpu().numpy(), a.ps, a.D))).to(x.dtype))
    if keys:  # keys of some two units: queries of half of one over the unit
        a.q.copy_((a.q.double().clamp(-4, 4) * 2.0 ** (125 - max(keys))).to(BF).to(dtype))
    a.call()
    out, lse, sm, conf = a.results()
    assert np.isfinite(out).all() and np.isfinite(lse).all()
    k, v, q = (x.double().cpu().numpy() for x in (a.k, a.v, a.q))
    G = a.hq // a.hkv
    half, w = (2.0 ** -8, 2.0 ** -8) if dtype is BF else (2.0 ** -24, 0.0)
    for b in range(len(n)):
        for i in range(n[b]):
            e, row = a.have[b] + i + 1, a.start_h[b] + i
            slots = np.arange(e)
            page = a.table_h[b, slots // a.ps]
            for h in range(a.hkv):
                kk, vv = (x[page, h, slots % a.ps] for x in (k, v))
                o, ls, ms, av, big = (x[0] for x in paged.attend(q[row, h * G:(h + 1) * G][None], kk, vv, a.pos_h[b, :e], e - 1, 0, 0,
                                                                 int(a.sw_h[b])))
                assert 0.5 < big.max() < 200
                err = ((D + 8) * big + 4 * e / 32 + 144) * 2.0 ** -24
                least = (3 * e + 8) * 2.0 ** -149 + (2.0 ** -134 if dtype is BF else 0)
                tol = ((2 * err[:, None] + w) * av) * (1 + half) + half * np.abs(o) + e * 2.0 ** -124 * np.abs(vv).max() + least
                heads = slice(h * G, (h + 1) * G)
                assert (np.abs(out[row, heads] - o) <= tol).all(), (b, i, h, np.abs(out[row, heads] - o).max(), tol.min())
                assert (np.abs(lse[row, heads] - ls) <= err + 2.0 ** -22 * (np.abs(ls) + big)).all(), (b, i, h)
                assert (np.abs(sm[row, heads] - ms) <= 2 * err * ms + e * 2.0 ** -126).all(), (b, i, h)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n", [1, 40])
@pytest.mark.parametrize("e", [60, 0, -60, -109, -110, -117])
def test_bits_of_float32_queries(e, n, D):
    """Each token sees its own slot alone and each query has one value, of 24 bits, where the key is one unit: the lse is the score,
    one product. The terms of a query hold what is not below 2^-133, so the score is off by at most 2^-133 of the key (nothing
    from 2^-110 on), by its scaling into and out of powers of two, four roundings of 2^-24, and by the log of a sum next to 1."""
    a = Attend4(F32, D, 4, 1, 16, [0], [n], window=1, seed=30, holes=False)
    at = a.r.randint(0, D, (a.T, 4))
    m = (2 ** 23 + a.r.randint(0, 2 ** 23, (a.T, 4))) * a.r.choice([-1, 1], (a.T, 4)) * 2.0 ** (e - 23)
    q = np.zeros((a.T, 4, D))
    np.put_along_axis(q, at[..., None], m[..., None], -1)
    a.q.copy_(torch.as_tensor(q.astype(np.float32)))
    x = 127 - e + 6  # scores of 64 to 128 over sqrt(D)
    block = fp4.pack(np.full(a.k.shape, 2, np.uint8), np.full((*a.k.shape[:-1], D // 32), x, np.uint8))
    a.bytes[0].copy_(torch.as_tensor(block))
    a.call()
    s = m[:n] * 2.0 ** (x - 127) / np.sqrt(D)
    lost = 2.0 ** -133 * 2.0 ** (x - 127) / np.sqrt(D) if e < -110 else 0
    lse = a.results()[1][:n]
    assert (np.abs(lse - s) <= 2.0 ** -21 * (np.abs(s) + 1) + lost).all(), np.abs(lse - s).max()
