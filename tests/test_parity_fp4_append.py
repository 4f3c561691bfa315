"""lg_rope_append_axes and lg_page_unpack_fp4 against oracle/fp4.py: queries, keys and values in pages of every type, rows
read back, and every byte that the calls have to leave alone.

Error of one rotated value scale (x cos a - y sin a): cos and sin are rounded once from double (2^-24; the angle's error
there, p f 2^-52, is below 2^-20 of that for the positions here), the products and the sum add 2^-24 each: under
4 x 2^-24 scale (|x| + |y|), or where sine and product are fused less. A stored type other than 4 bits adds half a
step. A value in 4 bits has to be the code nearest to some number within that error of the exact one, in a unit that
belongs to some largest magnitude within it."""
import numpy as np
import pytest
import torch

from oracle import fp4

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32
HALF_STEP = {BF: 2.0 ** -8, F32: 2.0 ** -24}


def near(x, tol, got, exps, what):
    """got (values), exps: 4-bit rows of numbers within tol of x."""
    n = x.shape[-1]
    group = lambda y: y.reshape(*y.shape[:-1], n // 32, 32)  # noqa: E731
    size, err = group(np.abs(x)), group(tol)
    low, high = fp4.exponent(np.maximum(size - err, 0).max(-1)), fp4.exponent((size + err).max(-1))
    assert ((exps >= low) & (exps <= high)).all(), what
    unit = np.repeat(2.0 ** (exps.astype(np.float64) - 127), 32, -1)
    ends = [np.sign(y) * fp4.STEPS[fp4.nearest(np.abs(y) / unit)] * unit for y in (x - tol, x + tol)]
    bad = ~((got >= ends[0]) & (got <= ends[1]))
    assert not bad.any(), (what, np.argwhere(bad)[:3], got[bad][:3], x[bad][:3])


class Step:
    """A map with room for n[b] new tokens behind have[b] slots, a projection's rows and the call's arrays."""

    def __init__(self, dtype, bits, D, hq, hkv, ps, have, n, axes=0, seed=0, far=0, extra=2, pad=0, gain=None):
        from paper_2604_10044_amd import lg
        self.lg, self.n, self.have, self.D, self.hq, self.hkv, self.ps = lg, n, have, D, hq, hkv, ps
        self.dtype, self.bits, self.axes = dtype, bits, axes
        r = np.random.RandomState(seed)
        B, P = len(n), max(-(-(h + x) // ps) for h, x in zip(have, n)) + 1
        n_pages = B * P + 3
        self.i32 = i32 = lambda x: torch.as_tensor(np.asarray(x, np.int32), device="cuda")  # noqa: E731
        self.table_h = r.permutation(n_pages)[:B * P].reshape(B, P)
        self.pos_h = far + np.arange(P * ps)[None] + r.randint(0, 50, (B, 1))
        self.table, self.pos = i32(self.table_h), i32(self.pos_h)
        self.len, self.ref = i32(np.add(have, n)), i32(np.ones(n_pages))
        g = torch.Generator(device="cuda").manual_seed(seed)
        if bits == 4:
            size = lg.fp4_page_bytes(ps, D)
            self.k, self.v = (torch.randint(0, 256, (n_pages, hkv, size), generator=g, device="cuda", dtype=torch.uint8) for _ in range(2))
            self.layer = lg.paged_layer_fp4(self.k, self.v, hq, ps, D)
        else:
            self.k, self.v = (torch.randn(n_pages, hkv, ps, D, generator=g, device="cuda").to(dtype) for _ in range(2))
            self.layer = lg.paged_layer(self.k, self.v, hq)
        self.map = lg.page_map(self.table, self.pos, self.len, self.ref, ps)
        self.total = sum(n) + extra  # rows behind the last sequence
        qkv = torch.randn(self.total, hq + 2 * hkv + pad, D, generator=g, device="cuda")
        if gain is not None:
            qkv *= 2.0 ** torch.randint(-gain, gain, (self.total, hq + 2 * hkv + pad, 1), generator=g, device="cuda").float()
        self.qkv = qkv.to(dtype)
        self.q, self.kn, self.vn = self.qkv[:, :hq], self.qkv[:, hq:hq + hkv], self.qkv[:, hq + hkv:hq + 2 * hkv]
        self.q_start, self.base = i32(np.concatenate([[0], np.cumsum(n)])), i32(have)
        self.out = torch.full((self.total, hq, D), 3.0, device="cuda", dtype=dtype)
        self.coord_h = r.randint(-300, 5000, (max(axes, 1), self.total)) + far
        self.coord = i32(self.coord_h) if axes else None

    def call(self, freq, rot, interleaved=False, scale=1.0, axis=None, q=True, kv=True, out=None, stream=None):
        self.axis_h = np.zeros(64, int) if axis is None else np.asarray(axis)
        self.lg.lg_rope_append_axes(
            self.layer, self.map, self.q if q else None, self.kn if kv else None, self.vn if kv else None, freq, rot, interleaved, scale,
            None if axis is None else self.i32(axis), None if axis is None else self.coord, (self.out if out is None else out) if q else None,
            self.q_start, self.base, stream=stream)

    def state(self):
        torch.cuda.synchronize()
        host = lambda x: x.cpu().numpy() if x.dtype is torch.uint8 else x.double().cpu().numpy()  # noqa: E731
        return [host(x) for x in (self.k, self.v, self.out, self.qkv)]

    def check(self, freq, rot, interleaved, scale, was, skip=(), kv=True, q=True):
        k, v, out, qkv = was
        got = self.state()
        f = np.zeros(64) if freq is None else freq.cpu().numpy()
        coord = self.coord_h if self.axes else np.zeros((1, self.total), int)
        rows, page, off, at = [], [], [], 0
        for b, n in enumerate(self.n):
            slots = self.have[b] + np.arange(n)
            if not self.axes:
                coord[0, at:at + n] = self.pos_h[b, slots]
            if b not in skip:
                rows += list(range(at, at + n))
                page += list(self.table_h[b, slots // self.ps])
                off += list(slots % self.ps)
            at += n
        rows, page, off = (np.asarray(x, int) for x in (rows, page, off))
        y, size = fp4.rope_axes(qkv[rows][:, :self.hq + self.hkv], coord[:, rows], np.minimum(np.maximum(self.axis_h, 0), max(self.axes, 1) - 1),
                                f, rot, interleaved, float(np.float32(scale)))
        tol = np.where(np.arange(self.D) < rot, 4 * 2.0 ** -24 * size, 0)
        half = HALF_STEP[self.dtype]
        want = out.copy()
        if q:
            want[rows] = y[:, :self.hq]
            err = np.zeros_like(out)
            err[rows] = tol[:, :self.hq] + np.where(np.arange(self.D) < rot, half * (np.abs(y) + tol)[:, :self.hq], 0)
            assert (np.abs(got[2] - want) <= err).all()
        else:
            np.testing.assert_array_equal(got[2], want)
        if not kv:
            rows = rows[:0]
        values = qkv[rows][:, self.hq + self.hkv:self.hq + 2 * self.hkv]
        y, tol = y[:len(rows), self.hq:], tol[:len(rows), self.hq:]
        page, off = page[:len(rows)], off[:len(rows)]
        if self.bits != 4:
            for x, now, new, err in ((k, got[0], y, tol + np.where(np.arange(self.D) < rot, half * (np.abs(y) + tol), 0)), (v, got[1], values, 0)):
                want, most = x.copy(), np.zeros_like(x)
                want[page, :, off], most[page, :, off] = new, err
                assert (np.abs(now - want) <= most).all()
            return
        for name, x, now, new, err in (("k", k, got[0], y, tol), ("v", v, got[1], values, np.zeros_like(values))):
            codes, exps = (z.copy() for z in fp4.unpack(x, self.ps, self.D))
            codes1, exps1 = fp4.unpack(now, self.ps, self.D)
            c, e = codes1[page, :, off], exps1[page, :, off]
            near(new, err, fp4.values(c, e), e, name)
            if name == "v":
                c0, e0 = fp4.encode(new)
                np.testing.assert_array_equal(e, e0)
                np.testing.assert_array_equal(fp4.values(c, e), fp4.values(c0, e0))
            codes[page, :, off], exps[page, :, off] = c, e  # everything else is as it was
            np.testing.assert_array_equal(now, fp4.pack(codes, exps))


def _freq(rot, theta=1e4):
    return torch.as_tensor((theta ** (-np.arange(0, rot, 2) / max(rot, 1))).astype(np.float32), device="cuda")


CASES = [
    # dtype, bits, D, hq, hkv, page, have, n
    (BF, 4, 128, 28, 4, 64, [0, 1, 63, 64, 200], [1, 1, 1, 1, 1]),
    (BF, 4, 64, 4, 4, 16, [0, 17, 3, 9], [40, 0, 33, 1]),
    (F32, 4, 128, 5, 1, 32, [100, 0], [2, 65]),
    (F32, 4, 64, 16, 2, 256, [250, 10], [70, 1]),
    (BF, 16, 128, 12, 2, 16, [5, 0], [20, 3]),
    (F32, 32, 64, 4, 4, 128, [127, 1], [2, 31]),
]


@pytest.mark.parametrize("axes", [0, 1, 2, 3, 8])
@pytest.mark.parametrize("dtype,bits,D,hq,hkv,ps,have,n", CASES)
def test_append(dtype, bits, D, hq, hkv, ps, have, n, axes):
    for rot, interleaved, scale in ((D, False, 1.0), (D, True, 1.125), (D // 2, False, 1.1386), (D // 2 + 16, True, 1.0), (36, False, 1.0),
                                    (50, True, 0.9), (2, False, 1.0), (2, True, 1.0), (0, False, 1.0)):
        s = Step(dtype, bits, D, hq, hkv, ps, have, n, axes=axes, seed=rot + axes)
        was = s.state()
        axis = None if axes == 0 else np.random.RandomState(rot).randint(0, axes, max(rot // 2, 1))
        f = _freq(rot) if rot else None
        s.call(f, rot, interleaved, scale, axis=axis)
        s.check(f, rot, interleaved, scale, was)


@pytest.mark.parametrize("bits", [4, 16])
def test_far_coordinates(bits):
    """Coordinates near 2^30, and below zero: angles keep their fraction of a turn. (2^30 turns are off by 2^-22 of one in
    double; 2 pi 2^-22 of the pair's size is added to the error.)"""
    s = Step(BF, bits, 128, 4, 2, 32, [3], [37], axes=3, seed=1, far=2 ** 30 - 10000)
    s.coord_h[1] = -s.coord_h[1]
    s.coord = s.i32(s.coord_h)
    was = s.state()
    f = _freq(128)
    s.call(f, 128, axis=s.lg.lg_rope_axes([20, 20, 24], s.lg.LG_AXES_TURNS).numpy())
    got = s.state()
    y, size = fp4.rope_axes(was[3][:37, :6], s.coord_h[:, :37], s.axis_h, f.cpu().numpy(), 128, False, 1.0)
    tol = (4 * 2.0 ** -24 + 2 * np.pi * 2.0 ** -22) * size
    assert (np.abs(got[2][:37] - y[:, :4]) <= (tol + 2.0 ** -8 * (np.abs(y) + tol))[:, :4]).all()
    if bits == 4:
        slots = 3 + np.arange(37)
        codes, exps = (x[s.table_h[0, slots // 32], :, slots % 32] for x in fp4.unpack(got[0], 32, 128))
        near(y[:, 4:], tol[:, 4:], fp4.values(codes, exps), exps, "far")


def test_axes_out_of_range_and_strides():
    """Axis numbers outside the axes count as the nearest; coordinates lie a stride apart; rows of a wider projection."""
    s = Step(BF, 4, 64, 4, 2, 16, [4, 0], [9, 30], axes=3, seed=2, pad=3)
    wide = torch.zeros(3, s.total + 11, dtype=torch.int32, device="cuda")
    wide[:, :s.total] = s.coord
    s.coord = wide
    was = s.state()
    axis = np.array([-5, 0, 1, 2, 3, 100, -1, 2] * 4)
    f = _freq(64)
    s.call(f, 64, True, axis=axis)
    s.check(f, 64, True, 1.0, was)


def test_values_of_every_size():
    """Heads from 2^-60 to 2^60, and with zeros alone."""
    for dtype in (BF, F32):
        s = Step(dtype, 4, 128, 4, 4, 16, [0, 3], [33, 20], seed=3, gain=60)
        s.kn[5] = 0
        s.vn[7, 1] = 0
        s.vn[8] = -0.0
        was = s.state()
        f = _freq(128)
        s.call(f, 128)
        s.check(f, 128, False, 1.0, was)


def test_ties_and_borders():
    """Values in the middle of two codes, and groups whose largest value is at the border of two units, float32 and the
    least and largest units."""
    steps = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0])
    near_ = np.concatenate([steps, np.nextafter(steps.astype(np.float32), np.float32(9)), np.nextafter(steps.astype(np.float32), np.float32(0)), -steps])
    s = Step(F32, 4, 64, 2, 2, 16, [0], [12], seed=4, extra=0)
    units = [0, 1, -7, 60, -100, -124, -125, -126, -130, 125, 124, 126]
    for i, e in enumerate(units):
        for h in range(2):
            row = near_[np.random.RandomState(i + 20 * h).permutation(32)].astype(np.float64)
            both = np.concatenate([row, row / np.abs(row).max() * [6.0, np.nextafter(np.float32(6), np.float32(9)), 3.0][i % 3]])
            x = np.minimum(np.maximum(both * 2.0 ** e, -3.4e38), 3.4e38)
            s.vn[i, h] = torch.as_tensor(x.astype(np.float32))
            s.kn[i, h] = s.vn[i, h]
    was = s.state()
    s.call(None, 0)
    s.check(None, 0, False, 1.0, was)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_values_that_are_not_finite(dtype):
    """A group with an infinity or NaN stands for NaN; its neighbours are as ever."""
    s = Step(dtype, 4, 128, 2, 2, 16, [0], [6], seed=5, extra=0)
    s.vn[0, 0, 3], s.vn[1, 1, 127], s.vn[2, 0, 40] = float("inf"), float("nan"), float("-inf")
    s.kn[3, 1, 70] = float("nan")
    was = s.state()
    s.call(None, 0)
    got = s.state()
    for x, rows in ((got[0], s.kn), (got[1], s.vn)):
        codes, exps = fp4.unpack(x, 16, 128)
        c, e = codes[s.table_h[0, 0], :, :6].swapaxes(0, 1), exps[s.table_h[0, 0], :, :6].swapaxes(0, 1)
        c0, e0 = fp4.encode(rows.double().cpu().numpy())
        np.testing.assert_array_equal(e, e0)
        np.testing.assert_array_equal(fp4.values(c, e), fp4.values(c0, e0))
    assert int((e == 255).sum()) == 3
    k, v = (torch.full((6, 2, 128), 9.0, device="cuda", dtype=dtype) for _ in range(2))
    s.lg.lg_page_unpack_fp4(s.layer, s.map, k, v, s.i32([0, 6]), s.base)
    np.testing.assert_array_equal(v.double().cpu().numpy(), fp4.values(c0, e0))
    assert int(k.isnan().sum()) == 32
    del was


def test_parts_alone():
    """Queries alone, keys and values alone, and queries in place."""
    for bits in (4, 16):
        f, axis = _freq(128), np.arange(64) % 3
        s = Step(BF, bits, 128, 8, 2, 32, [7, 0], [9, 40], axes=3, seed=6)
        was = s.state()
        s.call(f, 128, axis=axis, kv=False)
        s.check(f, 128, False, 1.0, was, kv=False)
        s = Step(BF, bits, 128, 8, 2, 32, [7, 0], [9, 40], axes=3, seed=6)
        s.call(f, 128, axis=axis, q=False)
        s.check(f, 128, False, 1.0, was, q=False)
        s = Step(BF, bits, 128, 8, 2, 32, [7, 0], [9, 40], axes=3, seed=6)
        s.q = s.out.copy_(s.q)
        s.call(f, 128, axis=axis)
        s.check(f, 128, False, 1.0, [was[0], was[1], s.qkv[:, :8].double().cpu().numpy(), was[3]])


def test_refused_sequences_and_missing_pages():
    """base < 0, a base that leaves no room and slots without a page: rows stay, pages stay."""
    for bits in (4, 32):
        s = Step(F32, bits, 64, 4, 2, 16, [5, 0, 3, 8], [7, 4, 5, 2], seed=7)
        s.base.copy_(s.i32([5, -1, 3, 10 ** 6]))
        s.table[2] = s.i32([-1, 10 ** 9] * 8)[:s.table.shape[1]]
        was = s.state()
        s.call(_freq(64), 64)
        s.check(_freq(64), 64, False, 1.0, was, skip={1, 2, 3})


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("D,hkv,ps", [(64, 1, 16), (128, 3, 64), (64, 8, 256)])
def test_unpack(dtype, D, hkv, ps):
    """Whole sequences and parts of them, any bytes; rows of refused sequences and missing pages stay."""
    from paper_2604_10044_amd import lg
    r = np.random.RandomState(D + ps)
    lens = [0, 1, ps, 3 * ps + 5, 40]
    B, P = len(lens), 5
    n_pages = B * P
    i32 = lambda x: torch.as_tensor(np.asarray(x, np.int32), device="cuda")  # noqa: E731
    k, v = (r.randint(0, 256, (n_pages, hkv, lg.fp4_page_bytes(ps, D))).astype(np.uint8) for _ in range(2))
    for x in (k, v):  # a third of the exponents are those of ordinary values, the others anything
        e = x[..., ps * D // 2:]
        e[r.rand(*e.shape) < 0.3] = 130
        # 4 and 6 units of 2^126 are no numbers of these types, and bytes 0 and 1 are units that the type's least normal
        # numbers do not reach by half a unit: neither is written by the append
        e[e < 2] = 2
    table = r.permutation(n_pages).reshape(B, P)
    table[3, 1] = -1
    kd, vd = torch.as_tensor(k, device="cuda"), torch.as_tensor(v, device="cuda")
    layer = lg.paged_layer_fp4(kd, vd, 2 * hkv, ps, D)
    m = lg.page_map(i32(table), i32(np.tile(np.arange(P * ps), (B, 1))), i32(lens), i32(np.ones(n_pages)), ps)
    start = np.concatenate([[0], np.cumsum(lens)])
    T = start[-1] + 2
    for base, both in ((np.zeros(B, int), True), (np.array([0, 4, 2, 7, -1]), False)):
        ko, vo = (torch.full((T, hkv, D), 9.0, device="cuda", dtype=dtype) for _ in range(2))
        lg.lg_page_unpack_fp4(layer, m, ko, vo if both else None, i32(start), i32(base))
        torch.cuda.synchronize()
        for x, o, asked in ((k, ko, True), (v, vo, both)):
            want = np.full((T, hkv, D), 9.0)
            val = fp4.values(*fp4.unpack(x, ps, D))
            for b, n in enumerate(lens):
                for i in range(n):
                    s = base[b] + i
                    if asked and base[b] >= 0 and table[b, s // ps] >= 0:
                        want[start[b] + i] = val[table[b, s // ps], :, s % ps]
            np.testing.assert_array_equal(o.double().cpu().numpy(), want)


@pytest.mark.parametrize("total", [2047, 2048, 5000, 9000, 30000])
def test_unpack_of_many_slots(total):
    """Batches whose workgroups read 1 to 16 slots each: sequences that begin and end inside one, empty ones, rows before the
    first and behind the last sequence, missing pages and refused sequences."""
    from paper_2604_10044_amd import lg
    r = np.random.RandomState(total)
    ps, hkv, D = 16, 2, 64
    lens = []
    while sum(lens) < total - 5:
        lens.append(int(min(r.choice([0, 1, 2, 5, 17, 100, 700]), total - 5 - sum(lens))))
    B, P = len(lens), max(1, -(-max(lens) // ps))
    pages = [-(-n // ps) for n in lens]
    table, at = np.full((B, P), -1), 0
    order = r.permutation(sum(pages) + 1)
    for b in range(B):
        table[b, :pages[b]] = order[at:at + pages[b]]
        at += pages[b]
    holes = (table >= 0) & (r.rand(B, P) < 0.02)
    table[holes] = r.choice([-1, 10 ** 9], int(holes.sum()))
    k, v = (r.randint(0, 256, (len(order), hkv, lg.fp4_page_bytes(ps, D))).astype(np.uint8) for _ in range(2))
    k[..., ps * D // 2:], v[..., ps * D // 2:] = 120, 130
    i32 = lambda x: torch.as_tensor(np.asarray(x, np.int32), device="cuda")  # noqa: E731
    layer = lg.paged_layer_fp4(torch.as_tensor(k, device="cuda"), torch.as_tensor(v, device="cuda"), hkv, ps, D)
    m = lg.page_map(i32(table), i32(np.zeros((B, P * ps))), i32(lens), i32(np.ones(len(order))), ps)
    start, base = 3 + np.concatenate([[0], np.cumsum(lens)]), np.where(r.rand(B) < 0.05, -1, 0)
    ko, vo = (torch.full((total, hkv, D), 9.0, device="cuda", dtype=F32) for _ in range(2))
    lg.lg_page_unpack_fp4(layer, m, ko, vo, i32(start), i32(base))
    torch.cuda.synchronize()
    seq = np.repeat(np.arange(B), lens)
    slot = np.concatenate([np.arange(n) for n in lens])
    page = table[seq, slot // ps]
    live = (base[seq] >= 0) & (page >= 0) & (page < len(order))
    for x, o in ((k, ko), (v, vo)):
        want = np.full((total, hkv, D), 9.0)
        val = fp4.values(*fp4.unpack(x, ps, D))
        want[3 + np.flatnonzero(live)] = val[page[live], :, slot[live] % ps]
        np.testing.assert_array_equal(o.double().cpu().numpy(), want)


def test_unpack_over_thousands_of_empty_sequences():
    """The rows of a workgroup belong to sequences far apart, or next to each other."""
    from paper_2604_10044_amd import lg
    B, ps, D, r = 40000, 16, 64, np.random.RandomState(3)
    lens = np.zeros(B, np.int64)
    some = np.unique(np.concatenate([r.randint(0, 3000, 700), r.randint(37000, B, 700), np.arange(2990, 3000)]))
    lens[some] = r.choice([1, 2, 3, 15, 16, 17, 60], len(some))
    total = int(lens.sum())
    assert total > 16 * 1024  # 16 slots a workgroup
    P = -(-int(lens.max()) // ps)
    P_of = -(-lens // ps)
    i32 = lambda y: torch.as_tensor(np.asarray(y, np.int32), device="cuda")  # noqa: E731
    pages, start = int(P_of.sum()), np.concatenate([[0], np.cumsum(lens)])
    order, off = r.permutation(pages), np.concatenate([[0], np.cumsum(P_of)])
    table = np.full((B, P), -1)
    for b in some:
        table[b, :P_of[b]] = order[off[b]:off[b + 1]]
    table = i32(table)
    x = r.randint(0, 256, (pages, 1, lg.fp4_page_bytes(ps, D))).astype(np.uint8)
    x[..., ps * D // 2:] = 127
    d = torch.as_tensor(x, device="cuda")
    layer = lg.paged_layer_fp4(d, d.clone(), 1, ps, D)
    m = lg.page_map(table, torch.zeros(B, P * ps, dtype=torch.int32, device="cuda"), i32(lens), i32(np.ones(pages)), ps)
    o = torch.full((total, 1, D), 9.0, device="cuda")
    lg.lg_page_unpack_fp4(layer, m, o, None, i32(start), i32(np.zeros(B)))
    seq = np.repeat(np.arange(B), lens)
    slot = np.arange(total) - start[seq]
    page = order[off[seq] + slot // ps]
    np.testing.assert_array_equal(o.double().cpu().numpy(), fp4.values(*fp4.unpack(x, ps, D))[page, :, slot % ps])


@pytest.mark.parametrize("bits", [4, 16])
def test_many_sequences(bits):
    """More sequences than a wave looks at together, some without tokens."""
    n = [(b * 7) % 4 for b in range(150)]
    s = Step(BF, bits, 64, 4, 2, 16, [(b * 5) % 30 for b in range(150)], n, axes=3, seed=11)
    was = s.state()
    f = _freq(64)
    s.call(f, 64, axis=np.arange(32) % 3)
    s.check(f, 64, False, 1.0, was)


def test_rows_before_the_first_sequence():
    """q_start need not begin at 0: rows before it are no sequence's."""
    s = Step(BF, 4, 64, 4, 2, 16, [4, 9], [7, 3], seed=12, extra=6)
    was = s.state()
    s.q_start.add_(5)
    f = _freq(64)
    s.call(f, 64)
    got = s.state()
    assert (got[2][:5] == 3).all() and (got[2][15:] == 3).all() and (got[2][5:15] != 3).any(-1).all()
    # the same as with the rows in front
    t = Step(BF, 4, 64, 4, 2, 16, [4, 9], [7, 3], seed=12, extra=6)
    t.qkv[:10] = s.qkv[5:15]
    t.call(f, 64)
    for x, y in zip(got[:2], t.state()[:2]):
        np.testing.assert_array_equal(x, y)
    np.testing.assert_array_equal(got[2][5:15], t.state()[2][:10])
    del was


def test_append_then_unpack_on_another_stream_and_in_a_graph():
    """An append and a read back, captured and replayed with other rows and places, against eager calls."""
    from paper_2604_10044_amd import lg
    f, axis = _freq(128), np.arange(64) % 3
    s = Step(BF, 4, 128, 8, 2, 32, [7, 0], [9, 40], axes=3, seed=8, extra=0)
    ax = s.i32(axis)
    k, v = (torch.zeros(49, 2, 128, device="cuda", dtype=BF) for _ in range(2))

    def step(stream=None):
        lg.lg_rope_append_axes(s.layer, s.map, s.q, s.kn, s.vn, f, 128, False, 1.0, ax, s.coord, s.out, s.q_start, s.base, stream=stream)
        lg.lg_page_unpack_fp4(s.layer, s.map, k, v, s.q_start, s.base, stream=stream)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    step(side)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for rep in range(4):
        s.qkv.normal_()
        s.coord.add_(17)
        step()
        torch.cuda.synchronize()
        want = [x.clone() for x in (s.k, s.v, s.out, k, v)]
        for x in (s.k, s.v, s.out, k, v):
            x.zero_()
        for x, y in ((s.k, want[0]), (s.v, want[1])):  # rows that the step does not write
            x.copy_(y)
        graph.replay()
        torch.cuda.synchronize()
        for x, y in zip((s.k, s.v, s.out, k, v), want):
            assert torch.equal(x, y)


def test_large_offsets():
    """Pages whose bytes lie beyond 2^32."""
    from paper_2604_10044_amd import lg
    n_pages, ps, hkv, D = 300000, 128, 2, 128  # 5.2 GB each of K and V
    s = Step(BF, 4, D, 4, hkv, ps, [100], [60], seed=9, extra=0)
    k = torch.zeros(n_pages, hkv, lg.fp4_page_bytes(ps, D), dtype=torch.uint8, device="cuda")
    v = torch.zeros_like(k)
    was = s.state()
    f = _freq(128)
    s.call(f, 128)
    pages = [299999, 255000, 7][:s.table.shape[1]]
    for c, p in enumerate(pages):
        k[p], v[p] = torch.as_tensor(was[0][s.table_h[0, c]], device="cuda"), torch.as_tensor(was[1][s.table_h[0, c]], device="cuda")
    m = lg.page_map(s.i32([pages]), s.pos, s.len, s.i32(np.ones(n_pages)), ps)
    layer = lg.paged_layer_fp4(k, v, 4, ps, D)
    out = torch.zeros_like(s.out)
    lg.lg_rope_append_axes(layer, m, s.q, s.kn, s.vn, f, 128, False, 1.0, None, None, out, s.q_start, s.base)
    torch.cuda.synchronize()
    assert torch.equal(out, s.out)
    for c, p in enumerate(pages):
        assert torch.equal(k[p], s.k[int(s.table_h[0, c])]) and torch.equal(v[p], s.v[int(s.table_h[0, c])])
    a, b = (torch.zeros(60, hkv, D, dtype=F32, device="cuda") for _ in range(2))
    c, d = torch.zeros_like(a), torch.zeros_like(a)
    lg.lg_page_unpack_fp4(layer, m, a, b, s.q_start, s.base)
    lg.lg_page_unpack_fp4(s.layer, s.map, c, d, s.q_start, s.base)
    assert torch.equal(a, c) and torch.equal(b, d) and float(a.abs().max()) > 0


def test_binding_refuses():
    from paper_2604_10044_amd import lg
    f, axis = _freq(64), np.arange(32) % 2
    s = Step(BF, 4, 64, 4, 2, 16, [4], [9], axes=2, seed=10, extra=0)
    was = s.state()
    for name, bad in (("q", s.q.float()), ("q", s.q[:, :3]), ("kn", s.kn[:-1]), ("vn", s.vn.float()), ("out", s.out[:-1]), ("coord", s.coord[:, :-1]),
                      ("coord", s.coord.long()), ("coord", s.coord.cpu()), ("coord", s.coord[0]), ("coord", None), ("base", s.base.long()),
                      ("q_start", s.q_start[:-1]), ("q", s.q.half()), ("kn", None)):
        keep = getattr(s, name)
        setattr(s, name, bad)
        with pytest.raises(lg.LGError):
            s.call(f, 64, axis=axis)
        setattr(s, name, keep)
    with pytest.raises(lg.LGError):
        s.call(f[:-1], 64, axis=axis)
    with pytest.raises(lg.LGError):
        s.call(f, 64, axis=axis[:-1])
    with pytest.raises(lg.LGError):
        lg.lg_rope_append(s.layer, s.map, s.q, s.kn, s.vn, f, 64, False, 1.0, s.out, s.q_start, s.base)
    k = torch.zeros(9, 2, 64, device="cuda", dtype=BF)
    for a, b in ((k, k.float()), (k[:-1], k), (k, k), (None, None), (k.half(), None)):
        with pytest.raises(lg.LGError):
            lg.lg_page_unpack_fp4(s.layer, s.map, a, b, s.q_start, s.base)
    s.call(f, 64, axis=axis)
    s.check(f, 64, False, 1.0, was)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("D", [64, 128])
def test_unpack_of_every_exponent_and_code(dtype, D):
    """Each of the 16 codes beside each exponent byte: the values are exact in both types, those below the least normal number
    too (2^-128 is the least), and bytes above 252 stand for NaN."""
    from paper_2604_10044_amd import lg
    ps, n_pages = 256, D // 32
    codes, exps = np.zeros((n_pages, 1, ps, D), np.uint8), np.zeros((n_pages, 1, ps, D // 32), np.uint8)
    for p in range(n_pages):  # the groups of a row have bytes far apart
        exps[p, 0] = (np.arange(ps)[:, None] + 64 * np.arange(D // 32) + p) % 256
        codes[p, 0] = (np.arange(D) + p) % 16
    pages = torch.as_tensor(fp4.pack(codes, exps), device="cuda")
    layer = lg.paged_layer_fp4(pages, pages.clone(), 1, ps, D)
    i32 = lambda x: torch.as_tensor(np.asarray(x, np.int32), device="cuda")  # noqa: E731
    m = lg.page_map(i32(np.arange(n_pages)[None]), i32(np.arange(n_pages * ps)[None]), i32([n_pages * ps]), i32(np.ones(n_pages)), ps)
    k, v = (torch.full((n_pages * ps, 1, D), 9.0, device="cuda", dtype=dtype) for _ in range(2))
    lg.lg_page_unpack_fp4(layer, m, k, v, i32([0, n_pages * ps]), i32([0]))
    want = fp4.values(codes, exps)[:, 0].reshape(-1, 1, D)
    assert 0 < np.nanmin(np.abs(want)[want != 0]) == 2.0 ** -128
    for x in (k, v):
        np.testing.assert_array_equal(x.double().cpu().numpy(), want)


@pytest.mark.parametrize("axes", [0, 3])
@pytest.mark.parametrize("far", [0, 2 ** 20, 2 ** 27, 2 ** 30 - 10000, 2 ** 31 - 10000])
def test_sines_are_rounded_once_at_any_distance(far, axes):
    """Pairs (1, 0) become (scale cos a, scale sin a) themselves, which are rounded once to float32: half a step of 2^-24
    beside what double leaves: the fraction of a turn is off by 2^-53 of one at most, 2 pi 2^-53, the sine and its product with
    scale by 2^-51 more. A coordinate times a frequency has up to 31 + 24 bits, so the fraction is not in its rounded product."""
    if axes == 0:
        far = min(far, 2 ** 30 - 10000)
    s = Step(F32, 32, 128, 4, 2, 32, [3, 0], [37, 41], axes=axes, seed=13, far=far)
    for x in (s.q, s.kn):
        x[..., :64], x[..., 64:] = 1, 0
    if axes:
        s.coord_h = np.random.RandomState(far % 1000).randint(far, far + 9000, s.coord_h.shape)
        s.coord_h[1] *= -1
        s.coord = s.i32(s.coord_h)
    was, freq = s.state(), _freq(128)
    axis = s.lg.lg_rope_axes([20, 20, 24], s.lg.LG_AXES_TURNS).numpy() if axes else None
    s.call(freq, 128, scale=1.25, axis=axis)
    got, T = s.state(), sum(s.n)
    coord = s.coord_h[:, :T] if axes else np.concatenate([s.pos_h[b, h:h + n] for b, (h, n) in enumerate(zip(s.have, s.n))])[None]
    want, _ = fp4.rope_axes(was[3][:T, :6], coord, s.axis_h, freq.cpu().numpy(), 128, False, 1.25)
    tol = 2.0 ** -24 * np.abs(want) + 1.25 * (2 * np.pi * 2.0 ** -53 + 2.0 ** -51)
    assert (np.abs(got[2][:T] - want[:, :4]) <= tol[:, :4]).all(), np.abs(got[2][:T] - want[:, :4]).max()
    slots = np.concatenate([h + np.arange(n) for h, n in zip(s.have, s.n)])
    k = got[0][s.table_h[np.repeat(np.arange(2), s.n), slots // 32], :, slots % 32]
    assert (np.abs(k - want[:, 4:]) <= tol[:, 4:]).all()
