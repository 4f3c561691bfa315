"""lg_page_reserve, lg_page_fork and lg_page_compact against the plain page map of oracle/paged.py: table,
positions, lengths, reference counts, base / moved and every row of every page, bit for bit (rows
that no sequence holds included: they are left as they were)."""
import numpy as np
import pytest
import torch

from oracle.paged import PageModel

pytestmark = pytest.mark.gpu


class Pool:
    """A paged cache on the device and its model beside it."""

    def __init__(self, B, P, ps, n_pages, L=2, Hkv=2, D=64, dtype=torch.bfloat16, seed=0, order=None):
        from paper_2604_10044_amd import lg
        self.lg, self.B, self.P, self.ps, self.cap = lg, B, P, ps, P * ps
        self.r = np.random.RandomState(seed)
        i32 = lambda x: torch.as_tensor(np.asarray(x, np.int32), device="cuda")  # noqa: E731
        self.i32 = i32
        self.table, self.pos = i32(np.full((B, P), -1)), i32(np.full((B, self.cap), -7))
        self.len, self.ref = i32(np.zeros(B)), i32(np.zeros(n_pages))
        rows = self.r.randint(0, 2 ** 15, (2 * L, n_pages, Hkv, ps, D)).astype(np.int16 if dtype == torch.bfloat16 else np.int32)
        self.kv = [torch.as_tensor(x, device="cuda").view(dtype) for x in rows]
        self.layers = [lg.paged_layer(self.kv[2 * i], self.kv[2 * i + 1], 2 * Hkv) for i in range(L)]
        self.map = lg.page_map(self.table, self.pos, self.len, self.ref, ps)
        self.ws = torch.empty(lg.lg_page_workspace(self.map), dtype=torch.uint8, device="cuda")
        self.ws.fill_(0xa5)
        self.base, self.moved = i32(np.full(B, 99)), i32(np.full(B, 99))
        self.model = PageModel(*(self.host(x) for x in (self.table, self.pos, self.len, self.ref)), ps, list(rows))

    def host(self, x):
        return x.cpu().numpy().copy()

    def bits(self, x):
        return x.view(torch.int16 if x.dtype == torch.bfloat16 else torch.int32).cpu().numpy()

    def check(self, what):
        torch.cuda.synchronize()
        m = self.model
        for name, x, y in (("len", self.len, m.len), ("table", self.table, m.table), ("pos", self.pos, m.pos),
                           ("ref", self.ref, m.ref)):
            np.testing.assert_array_equal(self.host(x), y, err_msg="%s: %s" % (what, name))
        for i, (x, y) in enumerate(zip(self.kv, m.kv)):
            np.testing.assert_array_equal(self.bits(x), y, err_msg="%s: kv %d" % (what, i))

    def reserve(self, n, t, what="reserve"):
        q = np.concatenate([[0], np.cumsum(n)])
        self.lg.lg_page_reserve(self.map, self.layers, self.i32(q), self.i32(t), self.base, self.ws)
        want = self.model.reserve(n, t)
        np.testing.assert_array_equal(self.host(self.base), want, err_msg=what)
        self.check(what)
        return want

    def fork(self, parent, what="fork"):
        self.lg.lg_page_fork(self.map, self.i32(parent), self.ws)
        self.model.fork(parent)
        self.check(what)

    def compact(self, keep, new_len, what="compact"):
        """keep: lists of kept slots, or None; pos and len are pruned as lg_prune_compact does."""
        nl = np.full(self.B, -1, np.int32)
        idx = self.r.randint(0, 2 ** 30, (self.B, self.cap)).astype(np.int32)  # entries behind new_len are not read
        for b, k in enumerate(keep):
            if k is not None:
                nl[b] = len(k)
                idx[b, :len(k)] = k
                for m in (self.model,):
                    m.pos[b, :len(k)] = m.pos[b, k]
                    m.len[b] = len(k)
        assert new_len is None
        self.pos.copy_(self.i32(self.model.pos))
        self.len.copy_(self.i32(self.model.len))
        self.lg.lg_page_compact(self.map, self.layers, self.i32(idx), self.i32(nl), self.moved, self.ws)
        want = self.model.compact(idx, nl)
        np.testing.assert_array_equal(self.host(self.moved), want, err_msg=what)
        self.check(what)
        return want


@pytest.mark.parametrize("ps", [16, 32, 64, 128, 256])
def test_reserve_lengths(ps):
    """Chunks of no token, one, a page less one, a page, a page and one, the whole cache."""
    p = Pool(7, 4, ps, 40, seed=ps)
    p.reserve([0, 1, ps - 1, ps, ps + 1, 4 * ps, 3], [5, 0, 100, 2000, 30000, 4 * ps - 1, 2 ** 30])
    p.reserve([0, 1, 1, 1, ps, 1, ps - 3], [5, 1, 101, 2001, 30000 + ps, 4 * ps, 2 ** 30 - 1])  # one is full
    p.reserve([3, 0, 0, 0, 0, 0, 0], [2, 0, 0, 0, 0, 0, 0])


def test_reserve_refuses_in_order():
    """With 6 free pages: what the first sequences need is met, the first that does not fit and every later one
    that needs a page are refused, one that needs none is served."""
    p = Pool(6, 8, 16, 6, seed=1)
    assert list(p.reserve([16, 1, 0, 0, 0, 0], [15, 0, 0, 0, 0, 0])) == [0, 0, 0, 0, 0, 0]
    base = p.reserve([16, 0, 17, 32, 1, 0], [31, 0, 16, 31, 0, 0])
    assert list(base) == [16, 1, 0, -1, -1, 0]
    base = p.reserve([8, 15, 8, 1, 0, 129], [39, 15, 24, 0, 0, 128])  # one page left, 129 beyond the columns
    assert list(base) == [32, 1, 17, -1, 0, -1]
    p.fork([-1] * 6)
    assert p.host(p.ref).sum() == 0


def test_reserve_at_the_edges_of_a_large_pool():
    """Free pages far apart: the search for them passes rounds of pages that are all held."""
    p = Pool(3, 300, 16, 20001, L=1, Hkv=1, seed=2)
    held = np.ones(20001, np.int32)
    held[[0, 4095, 4096, 8191, 12000, 20000]] = 0
    p.ref.copy_(p.i32(held))
    p.model.ref = held.copy()
    base = p.reserve([33, 32, 17], [32, 31, 16])
    assert list(base) == [0, 0, -1]
    assert list(p.model.table[0, :3]) == [0, 4095, 4096] and list(p.model.table[1, :2]) == [8191, 12000]
    p.reserve([0, 0, 16], [0, 0, 15])
    assert p.model.table[2, 0] == 20000


def test_many_sequences():
    """More sequences than the deciding workgroup has threads, one token each."""
    B = 1500
    p = Pool(B, 2, 16, 1400, L=1, Hkv=1, seed=3)
    base = p.reserve([1] * B, list(range(B)))
    assert (base[:1400] == 0).all() and (base[1400:] == -1).all()
    parent = np.arange(B)
    parent[::3] = np.arange(B)[::-1][::3]
    p.fork(parent)
    p.compact([[0] if b % 7 == 0 and p.model.len[b] else None for b in range(B)], None)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_forked_sequences_part(dtype):
    """Four samples of one prompt that ends inside a page: all of them copy it when they append, the page
    itself is free then; a fork that appends nothing keeps it."""
    p = Pool(5, 6, 16, 40, L=3, Hkv=3, D=128, dtype=dtype, seed=4)
    p.reserve([37, 0, 0, 0, 0], [36, 0, 0, 0, 0])
    p.fork([0, 0, 0, 0, 0])
    assert (p.model.ref[:3] == 5).all()
    p.reserve([1, 2, 20, 0, 1], [37, 38, 56, 0, 37])
    assert p.model.ref[2] == 1 and p.model.table[3, 2] == 2
    p.reserve([1, 1, 1, 1, 1], [38, 39, 57, 37, 38])  # now every last page is its own
    p.fork([-1, -1, -1, -1, 2])
    p.fork([4, 4, -1, 7, -5])  # 7 and -5 leave their sequences as they are


def test_fork_permutes():
    p = Pool(6, 4, 16, 30, seed=5)
    p.reserve([1, 16, 17, 33, 0, 64], [0, 15, 16, 32, 0, 63])
    p.fork([5, 4, 3, 2, 1, 0])
    p.fork([1, 2, 3, 4, 5, 0])
    p.fork([0, 1, 2, 3, 4, 5])


@pytest.mark.parametrize("P, lengths", [(64, [1024, 1023, 1025, 16384, 0]), (300, [76800, 65537, 65536, 1, 16640])])
def test_fork_of_long_sequences(P, lengths):
    """Rows that several workgroups copy, and more of them than the largest grid takes at once."""
    p = Pool(5, P, 256, sum((n + 255) // 256 for n in lengths) + 1, L=1, Hkv=1, seed=8)
    p.reserve(lengths, [n - 1 for n in lengths])
    p.fork([3, 0, 2, 1, 0])
    p.fork([1, 2, 0, -1, 3])


def test_compact_in_place_and_shared():
    p = Pool(6, 8, 16, 70, L=2, Hkv=2, D=128, seed=6)
    p.reserve([128, 100, 77, 16, 5, 0], [127, 99, 76, 15, 4, 0])
    every = lambda n, s, a=0: list(range(a)) + list(range(a, n, s))  # noqa: E731
    p.compact([every(128, 2, 20), None, every(77, 3), list(range(16)), [], None], None)
    # identical keep sets move nothing; keeping nothing frees everything
    p.compact([None, list(range(100)), [0], [15], None, None], None)
    p.fork([1, 1, 1, 3, 1, 1])
    # all share: the prefix that stays is still shared, the rest becomes everybody's own
    p.compact([every(100, 2, 40), every(100, 2, 40), every(100, 3, 16), None, list(range(50)), None], None)
    p.compact([list(range(30)), None, None, None, None, every(100, 5)], None)


def test_compact_refuses_without_pages():
    """Replacing shared pages needs free ones: the first sequence gets them, the second is refused and left as
    it was, the third needs none; after pages are freed the call is repeated for the refused one."""
    p = Pool(4, 4, 16, 10, seed=7)
    p.reserve([64, 0, 64, 0], [63, 0, 63, 0])
    p.fork([0, 0, 2, 0])  # 8 pages held, 2 free
    keep = [list(range(1, 30)), list(range(2, 40)), list(range(3, 64)), None]
    before = p.model.table.copy()
    assert list(p.compact(keep, None)) == [1, -1, 1, 0]
    np.testing.assert_array_equal(p.model.table[1], before[1])
    p.fork([-1, 1, -1, -1])
    nl = np.array([-1, 38, -1, -1], np.int32)
    idx = np.zeros((4, 64), np.int32)
    idx[1, :38] = np.arange(2, 40)
    p.lg.lg_page_compact(p.map, p.layers, p.i32(idx), p.i32(nl), p.moved, p.ws)
    assert list(p.model.compact(idx, nl)) == [0, 1, 0, 0]
    p.check("repeated")


@pytest.mark.parametrize("seed", range(6))
def test_random_histories(seed):
    """Steps, forks, ends and prunes of a batch on a pool that runs short now and then."""
    r = np.random.RandomState(seed)
    ps = int(r.choice([16, 32, 64]))
    B, P = int(r.randint(2, 9)), int(r.randint(3, 9))
    p = Pool(B, P, ps, int(B * P * 0.7) + 2, L=int(r.randint(1, 4)), Hkv=int(r.randint(1, 4)), D=int(r.choice([64, 128])),
             dtype=torch.bfloat16 if seed % 2 else torch.float32, seed=seed)
    t = np.full(B, -1)
    for step in range(40):
        what = "step %d" % step
        kind = r.choice(["reserve", "reserve", "reserve", "fork", "compact"])
        if kind == "reserve":
            n = r.choice([0, 1, 1, 1, 2, ps, 3 * ps // 2], B)
            want = p.reserve(n, t + n + r.randint(0, 5), what)
            live = np.maximum(p.model.len, 1) - 1
            t = np.where(want >= 0, p.model.pos[np.arange(B), live], t)
        elif kind == "fork":
            parent = np.arange(B)
            for b in r.choice(B, int(r.randint(1, B + 1)), replace=False):
                parent[b] = r.randint(-1, B)
            t = np.where((parent >= 0), t[np.maximum(parent, 0)], -1)
            p.fork(parent, what)
        else:
            keep = []
            for b in range(B):
                n = int(p.model.len[b])
                k = np.flatnonzero(r.rand(n) < r.choice([0.3, 0.8, 1.0]))
                if r.rand() < 0.5:
                    k = np.unique(np.concatenate([np.arange(n // 2), k])).astype(int)
                keep.append(list(k) if r.rand() < 0.5 else None)
            p.compact(keep, None, what)
        if kind != "compact" or (p.host(p.moved) >= 0).all():
            np.testing.assert_array_equal(p.model.ref, p.model.counted(), err_msg=what)
        else:
            # a refused sequence is ended, as a server without pages would
            parent = np.arange(B)
            parent[p.host(p.moved) < 0] = -1
            t = np.where(parent < 0, -1, t)
            p.fork(parent, what)


def test_map_alone():
    """No layers: the map's numbers change, no row moves."""
    p = Pool(3, 4, 16, 20, seed=8)
    layers, p.layers, p.model.kv = p.layers, [], []
    kv, p.kv = p.kv, []
    before = [p.bits(x).copy() for x in kv]
    p.reserve([40, 3, 0], [39, 2, 0])
    p.fork([0, 0, 1])
    p.reserve([1, 1, 1], [40, 40, 3])
    p.compact([list(range(20, 41)), None, None], None)
    for x, y in zip(kv, before):
        np.testing.assert_array_equal(p.bits(x), y)
    assert len(layers) == 2


def test_more_layers_than_a_launch_takes():
    p = Pool(2, 3, 16, 12, L=66, Hkv=1, D=64, seed=9)
    p.reserve([20, 0], [19, 0])
    p.fork([0, 0])
    p.reserve([1, 1], [20, 20])
    p.compact([list(range(1, 21)), list(range(0, 21, 2))], None)


def test_broken_values_stay_inside():
    """Values outside their ranges: nothing outside the arrays is touched, other sequences are served."""
    p = Pool(5, 4, 16, 20, seed=10)
    p.reserve([20, 20, 20, 20, 20], [19] * 5)
    guard = [x.clone() for x in p.kv]
    tab = p.host(p.table)
    tab[1] = [10 ** 9, -10 ** 9, 20, -1]
    p.table.copy_(p.i32(tab))
    p.len.copy_(p.i32([20, 20, 10 ** 9, -5, 20]))
    q = p.i32([0, 1, 2, 3, 3, 2])  # the last sequence's rows do not ascend
    p.lg.lg_page_reserve(p.map, p.layers, q, p.i32([20] * 5), p.base, p.ws)
    torch.cuda.synchronize()
    base = p.host(p.base)
    assert base[0] == 20 and base[1] == -1 and base[2] == -1 and base[3] == 0 and base[4] == 20
    keep = p.i32(np.full((5, 64), 2 ** 31 - 1))
    p.lg.lg_page_compact(p.map, p.layers, keep, p.i32([5, 2 ** 31 - 1, -9, 7, 3]), p.moved, p.ws)
    p.lg.lg_page_fork(p.map, p.i32([2 ** 31 - 1, -2 ** 31, 0, 1, 4]), p.ws)
    torch.cuda.synchronize()
    for x, y in zip(p.kv, guard):  # no source was inside, so no row has moved
        assert torch.equal(x.view(torch.int16), y.view(torch.int16))
