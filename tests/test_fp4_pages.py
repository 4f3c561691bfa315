"""lg_page_reserve, lg_page_fork and lg_page_compact on 4-bit layers against the plain page map of oracle/paged.py: every byte
of every page (rows that no sequence holds included: they are left as they were)."""
import numpy as np
import pytest
import torch

from oracle import fp4
from test_parity_pages import Pool

pytestmark = pytest.mark.gpu


class Pool4(Pool):
    """The model follows a row's codes and exponents side by side."""

    def __init__(self, B, P, ps, n_pages, L=2, Hkv=2, D=64, seed=0):
        super().__init__(B, P, ps, n_pages, L=1, Hkv=1, D=64, seed=seed)
        self.D = D
        raw = self.r.randint(0, 256, (2 * L, n_pages, Hkv, self.lg.fp4_page_bytes(ps, D))).astype(np.uint8)
        self.kv = [torch.as_tensor(x, device="cuda") for x in raw]
        self.layers = [self.lg.paged_layer_fp4(self.kv[2 * i], self.kv[2 * i + 1], 2 * Hkv, ps, D) for i in range(L)]
        self.model.kv = [np.concatenate(fp4.unpack(x, ps, D), -1) for x in raw]

    def bits(self, x):
        return np.concatenate(fp4.unpack(x.cpu().numpy(), self.ps, self.D), -1)


@pytest.mark.parametrize("ps,D,Hkv,L", [(16, 64, 2, 3), (16, 128, 3, 2), (64, 128, 1, 2), (256, 64, 2, 1), (32, 128, 8, 70)])
def test_forked_sequences_part_and_are_pruned(ps, D, Hkv, L):
    """A shared last page is copied, pruned rows move in place and to fresh pages, pages are given back."""
    p = Pool4(5, 6, ps, 40, L=L, Hkv=Hkv, D=D, seed=ps + D)
    first = 2 * ps + ps // 2 + 1
    p.reserve([first, 0, 5 * ps, 1, 0], [first - 1, 0, 5 * ps - 1, 0, 0])
    p.fork([0, 0, 2, 3, 2])
    p.reserve([3, 1, 1, 1, ps], [first + 2, first, 5 * ps, 1, 6 * ps - 1])
    lens = p.model.len.copy()
    keep = [None] * 5
    keep[0] = sorted(p.r.choice(lens[0], lens[0] // 2, replace=False))
    keep[2] = [0, 1] + list(range(5, lens[2] - 3, 2))
    keep[3] = [1]
    keep[4] = list(range(0, lens[4], 3))
    p.compact(keep, None)
    p.reserve([1, 1, 1, 1, 1], p.model.pos[np.arange(5), p.model.len - 1] + 1)
    p.compact([None, list(range(p.model.len[1] - 1)), None, None, []], None)


def test_long_histories_move_in_place():
    """Rows of several passes of a workgroup and several segments, in place."""
    for D in (64, 128):
        p = Pool4(2, 40, 128, 90, L=2, Hkv=2, D=D, seed=D)
        p.reserve([5000, 4000], [4999, 3999])
        keep = np.sort(p.r.choice(np.arange(7, 5000), 4300, replace=False))
        p.compact([list(range(7)) + list(keep), list(range(1, 4000))], None)


@pytest.mark.parametrize("seed", range(4))
def test_random_histories(seed):
    r = np.random.RandomState(seed)
    ps, B = [16, 32, 16, 64][seed], 6
    p = Pool4(B, 8, ps, 30, L=2, Hkv=1 + seed % 2, D=[64, 128][seed % 2], seed=seed)
    for step in range(12):
        n = r.randint(0, 2 * ps, B) * (r.rand(B) < 0.6)
        newest = [p.model.pos[b, p.model.len[b] - 1] if p.model.len[b] else -1 for b in range(B)]
        p.reserve(list(n), [int(t + x) for t, x in zip(newest, n)], "reserve %d" % step)
        if step % 3 == 1:
            p.fork([int(r.choice([b, b, r.randint(0, B), -1])) for b in range(B)], "fork %d" % step)
        if step % 3 == 2:
            keep = []
            for b in range(B):
                m = p.model.len[b]
                keep.append(sorted(r.choice(m, r.randint(0, m), replace=False)) if m and r.rand() < 0.5 else None)
            moved = p.compact(keep, None, "compact %d" % step)
            for b in np.flatnonzero(moved < 0):  # refused: ended, as its positions name other rows
                p.fork([-1 if x == b else x for x in range(B)], "end %d" % step)
