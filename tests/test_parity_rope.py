"""lg_rope_append against the rotation in 64 bits (oracle/paged.py): queries, the keys and values in their
pages, and every row that the call has to leave alone.

Error of one rotated value scale (x cos a - y sin a): the angle's fraction of a turn is rounded to
float32 (2^-26 turns at most, 2 pi 2^-26 < 2^-23 in the angle), sincospi adds 2 ulp (2^-23) and the scale
one rounding (2^-24): 2.5 x 2^-23 on each of cos and sin; the two products and their sum add 2 x 2^-24.
Together under 7 x 2^-24 scale (|x| + |y|), and half a step of the stored type."""
import numpy as np
import pytest
import torch

from oracle import paged

pytestmark = pytest.mark.gpu

HALF_STEP = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}


class Step:
    """A map with room for n[b] new tokens behind have[b] slots, a projection's rows and the call's arrays."""

    def __init__(self, dtype, D, hq, hkv, ps, have, n, seed=0, far=0, extra=2, gap=1, pad=0):
        from paper_2604_10044_amd import lg
        self.lg, self.n, self.have, self.D, self.hq, self.hkv, self.ps, self.dtype = lg, n, have, D, hq, hkv, ps, dtype
        r = np.random.RandomState(seed)
        B, P = len(n), max(-(-(h + x) // ps) for h, x in zip(have, n)) + 1
        n_pages = B * P + 3
        i32 = lambda x: torch.as_tensor(np.asarray(x, np.int32), device="cuda")  # noqa: E731
        self.i32 = i32
        self.table_h = r.permutation(n_pages)[:B * P].reshape(B, P)
        self.pos_h = far + gap * np.arange(P * ps)[None] + r.randint(0, 50, (B, 1))
        self.table, self.pos = i32(self.table_h), i32(self.pos_h)
        self.len, self.ref = i32(np.add(have, n)), i32(np.ones(n_pages))
        g = torch.Generator(device="cuda").manual_seed(seed)
        rand = lambda *s: torch.randn(*s, generator=g, device="cuda").to(dtype)  # noqa: E731
        self.k, self.v = rand(n_pages, hkv, ps, D), rand(n_pages, hkv, ps, D)
        self.total = sum(n) + extra  # rows behind the last sequence
        qkv = rand(self.total, hq + 2 * hkv + pad, D)
        self.qkv = qkv
        self.q, self.kn, self.vn = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:hq + 2 * hkv]
        self.q_start, self.base = i32(np.concatenate([[0], np.cumsum(n)])), i32(have)
        self.out = torch.full((self.total, hq, D), 3.0, device="cuda", dtype=dtype)
        self.layer = lg.paged_layer(self.k, self.v, hq)
        self.map = lg.page_map(self.table, self.pos, self.len, self.ref, ps)

    def call(self, freq, rot, interleaved, scale, q=None, out=None, kv=True, stream=None):
        self.lg.lg_rope_append(self.layer, self.map, self.q if q is None else q, self.kn if kv else None,
                               self.vn if kv else None, freq, rot, interleaved, scale,
                               self.out if out is None else out, self.q_start, self.base, stream=stream)

    def check(self, freq, rot, interleaved, scale, was, got, kv=True, skip=()):
        """was: (q, kn, vn, k, v, out) before the call; got: (k, v, out) after it, all on the host."""
        q, kn, vn, k, v, out = was
        want_k, size_k = k.copy(), np.zeros_like(k)
        want_v = v.copy()
        want_q, size_q = out.copy(), np.zeros_like(out)
        at = 0
        for b, n in enumerate(self.n):
            rows, slots = np.arange(at, at + n), self.have[b] + np.arange(n)
            at += n
            if b in skip:
                continue
            p = self.pos_h[b, slots]
            want_q[rows], size_q[rows] = paged.rope(q[rows], p, freq, rot, interleaved, scale)
            if kv:
                y, size = paged.rope(kn[rows], p, freq, rot, interleaved, scale)
                page, off = self.table_h[b, slots // self.ps], slots % self.ps
                want_k[page, :, off], size_k[page, :, off] = y, size
                want_v[page, :, off] = vn[rows]
        half = HALF_STEP[self.dtype]
        for name, x, y, size in (("q", got[2], want_q, size_q), ("k", got[0], want_k, size_k)):
            tol = np.where(size > 0, 7 * 2.0 ** -24 * size + half * (np.abs(y) + 7 * 2.0 ** -24 * size), 0)
            bad = ~(np.abs(x - y) <= tol)
            assert not bad.any(), (name, np.argwhere(bad)[:3], np.abs(x - y).max())
        np.testing.assert_array_equal(got[1], want_v)


def _f64(*xs):
    return [x.double().cpu().numpy() for x in xs]


def _freq(rot, theta=1e4):
    return (theta ** (-np.arange(0, rot, 2) / max(rot, 1))).astype(np.float32)


CASES = [
    # dtype, D, hq, hkv, page, have, n, rot, interleaved
    (torch.bfloat16, 128, 28, 4, 64, [0, 63, 64, 100], [1, 1, 1, 1], 128, False),
    (torch.bfloat16, 128, 28, 4, 64, [0, 63, 64, 100], [1, 1, 1, 1], 128, True),
    (torch.bfloat16, 64, 4, 4, 16, [0, 15, 3, 0, 7], [33, 2, 0, 16, 1], 64, False),
    (torch.float32, 64, 12, 2, 16, [5, 0], [40, 17], 64, True),
    (torch.float32, 128, 16, 1, 32, [31, 1, 0], [3, 70, 0], 128, False),
    (torch.bfloat16, 128, 6, 2, 128, [127, 0], [2, 5], 64, False),   # half of the head
    (torch.bfloat16, 128, 6, 2, 256, [250, 0], [9, 5], 96, True),
    (torch.bfloat16, 64, 3, 3, 16, [0, 9], [5, 8], 8, False),        # halves that are no whole pieces
    (torch.bfloat16, 64, 3, 3, 16, [0, 9], [5, 8], 24, False),
    (torch.bfloat16, 64, 3, 3, 16, [0, 9], [5, 8], 20, True),
    (torch.float32, 64, 2, 1, 16, [0, 9], [5, 8], 2, False),
    (torch.float32, 64, 2, 1, 16, [0, 9], [5, 8], 62, True),
    (torch.bfloat16, 128, 8, 8, 16, [2], [300], 0, False),           # no rotation: the append alone
]


@pytest.mark.parametrize("dtype,D,hq,hkv,ps,have,n,rot,ilv", CASES)
def test_rotation(dtype, D, hq, hkv, ps, have, n, rot, ilv):
    s = Step(dtype, D, hq, hkv, ps, have, n, seed=rot + D, pad=1)
    f = _freq(rot)
    was = _f64(s.q, s.kn, s.vn, s.k, s.v, s.out)
    for scale in (1.0, 1.25):
        s.call(torch.as_tensor(f, device="cuda") if rot else None, rot, ilv, scale)
        torch.cuda.synchronize()
        s.check(f, rot, ilv, scale, was, _f64(s.k, s.v, s.out))


@pytest.mark.parametrize("far", [10 ** 5, 10 ** 7, 2 ** 30 - 4000])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_far_positions(dtype, far):
    s = Step(dtype, 128, 4, 2, 16, [0, 700], [50, 3], seed=3, far=far, gap=1)
    f = _freq(128)
    was = _f64(s.q, s.kn, s.vn, s.k, s.v, s.out)
    s.call(torch.as_tensor(f, device="cuda"), 128, False, 1.0)
    s.check(f, 128, False, 1.0, was, _f64(s.k, s.v, s.out))


@pytest.mark.parametrize("rot,ilv", [(128, False), (128, True), (36, False), (36, True)])
def test_in_place_queries(rot, ilv):
    s = Step(torch.bfloat16, 128, 8, 2, 16, [4, 0], [20, 9], seed=5)
    f = _freq(rot)
    q = s.q.contiguous()
    was = _f64(q, s.kn, s.vn, s.k, s.v, q)
    s.call(torch.as_tensor(f, device="cuda"), rot, ilv, 1.0, q=q, out=q)
    s.check(f, rot, ilv, 1.0, was, _f64(s.k, s.v, q))


def test_queries_alone():
    s = Step(torch.bfloat16, 64, 8, 2, 16, [4, 0], [20, 9], seed=6)
    f = _freq(64)
    was = _f64(s.q, s.kn, s.vn, s.k, s.v, s.out)
    s.call(torch.as_tensor(f, device="cuda"), 64, False, 1.0, kv=False)
    s.check(f, 64, False, 1.0, was, _f64(s.k, s.v, s.out), kv=False)


def test_refused_and_broken_rows_are_left_alone():
    """A refused sequence, a slot behind the last column, and a missing page: their rows stay."""
    s = Step(torch.bfloat16, 64, 4, 2, 16, [4, 0, 3, 2, 5], [20, 9, 4, 5, 1], seed=7)
    f = _freq(64)
    base, table = [4, -1, 10 ** 9, 2, 5], s.table_h.copy()
    table[3] = [10 ** 9, -1, -1][:1] * table.shape[1]
    s.base.copy_(s.i32(base))
    s.table.copy_(s.i32(table))
    was = _f64(s.q, s.kn, s.vn, s.k, s.v, s.out)
    s.call(torch.as_tensor(f, device="cuda"), 64, False, 1.0)
    s.check(f, 64, False, 1.0, was, _f64(s.k, s.v, s.out), skip=(1, 2, 3))


def test_many_sequences_and_empty_ones():
    n = [(b * 7) % 3 for b in range(200)]
    s = Step(torch.bfloat16, 64, 2, 1, 16, [b % 40 for b in range(200)], n, seed=8)
    f = _freq(64)
    was = _f64(s.q, s.kn, s.vn, s.k, s.v, s.out)
    s.call(torch.as_tensor(f, device="cuda"), 64, True, 1.0)
    s.check(f, 64, True, 1.0, was, _f64(s.k, s.v, s.out))


def test_another_stream():
    s = Step(torch.bfloat16, 128, 8, 2, 16, [4, 0], [20, 9], seed=9)
    f = torch.as_tensor(_freq(128), device="cuda")
    was = _f64(s.q, s.kn, s.vn, s.k, s.v, s.out)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    s.call(f, 128, False, 1.0, stream=st)
    st.synchronize()
    s.check(_freq(128), 128, False, 1.0, was, _f64(s.k, s.v, s.out))


def test_binding_refuses():
    from paper_2604_10044_amd import lg
    s = Step(torch.bfloat16, 64, 4, 2, 16, [4, 0], [20, 9], seed=10)
    f = torch.as_tensor(_freq(64), device="cuda")
    bad = [dict(q=s.q.float()), dict(q=s.q[:, :3]), dict(out=s.out[:-1]), dict(out=s.out.float()),
           dict(q=s.q.cpu()), dict(q=s.q.transpose(1, 2))]
    for kw in bad:
        with pytest.raises(lg.LGError):
            s.call(f, 64, False, 1.0, **kw)
    with pytest.raises(lg.LGError):
        s.call(f[:31], 64, False, 1.0)
    with pytest.raises(lg.LGError):
        s.call(f, 66, False, 1.0)
    with pytest.raises(lg.LGError):
        lg.lg_rope_append(s.layer, s.map, s.q, s.kn, None, f, 64, False, 1.0, s.out, s.q_start, s.base)
    with pytest.raises(lg.LGError):
        lg.lg_rope_append(s.layer, s.map, s.q, s.kn[:-1], s.vn[:-1], f, 64, False, 1.0, s.out, s.q_start, s.base)
