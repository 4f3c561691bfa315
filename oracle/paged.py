"""Plain float64 / Python models of the paged cache's operators (include/lg_paged.h), written from their
definitions and sharing no code with the kernels: the page map as lists, sequence after sequence;
rotation and attention in numpy, token after token."""
from __future__ import annotations

import math

import numpy as np


class PageModel:
    """The page map of lg_paged.h as Python lists. Rows of a layer's K and V are followed through
    `kv`, arrays [n_pages][Hkv][page_size][D] changed in place."""

    def __init__(self, table, pos, len_, ref, page_size, kv=()):
        self.table, self.pos = table.copy(), pos.copy()
        self.len, self.ref = len_.copy(), ref.copy()
        self.ps, self.kv = page_size, [x.copy() for x in kv]
        self.B, self.P = table.shape
        self.cap = self.P * page_size

    def _pages(self, n):
        return -(-n // self.ps)

    def _serve(self, needs):
        """Which sequences' page needs are met, in order: none that needs a page after the first
        that what is free does not cover."""
        free, ok, short = int((self.ref == 0).sum()), [], False
        for need in needs:
            if need and (short or need > free):
                short = True
            else:
                free -= need
            ok.append(not (need and short))
        return ok

    def _take(self):
        p = int(np.flatnonzero(self.ref == 0)[0])
        return p

    def reserve(self, n_new, t):
        base = np.full(self.B, -1, np.int32)
        needs, able, shared = [], [], []
        for b in range(self.B):
            old, n = int(self.len[b]), int(n_new[b])
            fits = old + n <= self.cap
            part = old % self.ps != 0 and n > 0
            copy = fits and part and self.ref[self.table[b, old // self.ps]] > 1
            able.append(fits)
            shared.append(copy)
            needs.append(self._pages(old + n) - self._pages(old) + copy if fits else 0)
        ok = self._serve(needs)
        was = [x.copy() for x in self.kv]
        gone = []
        for b in range(self.B):
            if not (able[b] and ok[b]):
                continue
            old, n = int(self.len[b]), int(n_new[b])
            base[b] = old
            for c in ([old // self.ps] if shared[b] else []) + list(range(self._pages(old), self._pages(old + n))):
                p = self._take()
                if shared[b] and c == old // self.ps:
                    src = self.table[b, c]
                    gone.append(src)
                    for x, y in zip(self.kv, was):
                        x[p, :, :old % self.ps] = y[src, :, :old % self.ps]
                self.table[b, c] = p
                self.ref[p] = 1
            self.pos[b, old:old + n] = t[b] - n + 1 + np.arange(n)
            self.len[b] = old + n
        for p in gone:
            self.ref[p] -= 1
        return base

    def fork(self, parent):
        was = (self.table.copy(), self.pos.copy(), self.len.copy())
        for b in range(self.B):
            p = int(parent[b])
            if p == b or not -1 <= p < self.B:
                continue
            self.len[b] = was[2][p] if p >= 0 else 0
            self.table[b] = was[0][p] if p >= 0 else -1
            if p >= 0:
                self.pos[b, :self.len[b]] = was[1][p, :self.len[b]]
        self.ref[:] = self.counted()

    def counted(self):
        """References of every page, counted from the table."""
        ref = np.zeros_like(self.ref)
        for p in self.table[self.table >= 0]:
            ref[p] += 1
        return ref

    def compact(self, keep, new_len):
        moved = np.zeros(self.B, np.int32)
        plans, needs, ref0 = [], [], self.ref.copy()
        for b in range(self.B):
            plan = []
            if new_len[b] >= 0:
                n = int(new_len[b])
                still = 0
                while still < n and keep[b, still] == still:
                    still += 1
                first = still // self.ps if still < n else self._pages(n)
                plan = list(range(first, self._pages(n)))
            plans.append(plan)
            needs.append(sum(int(ref0[self.table[b, c]] > 1) for c in plan))
        ok = self._serve(needs)
        was, kv = self.table.copy(), [x.copy() for x in self.kv]
        gone = []
        for b in range(self.B):
            if new_len[b] < 0:
                continue
            moved[b] = 1 if ok[b] else -1
            if not ok[b]:
                continue
            n = int(new_len[b])
            for c in plans[b]:
                if ref0[was[b, c]] > 1:
                    p = self._take()
                    gone.append(was[b, c])
                    self.table[b, c], self.ref[p] = p, 1
            for c in range(self._pages(n), self.P):
                if was[b, c] >= 0:
                    gone.append(was[b, c])
                self.table[b, c] = -1
            for r in range(plans[b][0] * self.ps if plans[b] else n, n):
                s = int(keep[b, r])
                for x, y in zip(self.kv, kv):
                    x[self.table[b, r // self.ps], :, r % self.ps] = y[was[b, s // self.ps], :, s % self.ps]
        for p in gone:
            self.ref[p] -= 1
        return moved


def rope(x, pos, inv_freq, rot, interleaved, scale):
    """x [T][H][D] rotated at positions pos [T], in float64; also the sums |x| + |y| that its rounding
    errors are proportional to."""
    y = x.astype(np.float64).copy()
    size = np.zeros_like(y)
    for j in range(rot // 2):
        a, b = (2 * j, 2 * j + 1) if interleaved else (j, j + rot // 2)
        ang = pos.astype(np.longdouble) * np.longdouble(np.float32(inv_freq[j]))
        c, s = np.cos(ang).astype(np.float64)[:, None], np.sin(ang).astype(np.float64)[:, None]
        u, w = x[..., a].astype(np.float64), x[..., b].astype(np.float64)
        y[..., a], y[..., b] = scale * (u * c - w * s), scale * (w * c + u * s)
        size[..., a] = size[..., b] = scale * (np.abs(u) + np.abs(w))
    return y, size


def attend(q, k, v, pos, base, window, n_sink, suffix_w, see=None):
    """One KV head of one sequence: q [n][G][D], k, v, pos over the slots; `see` [slots] False hides
    a slot from every token. Returns float64 out [n][G][D], lse, mass [n][G], and for the error bounds
    sum alpha |v| [n][G][D] and the largest sum_d |q_d k_d| / sqrt(D) over the visible slots [n][G]."""
    n, G, D = q.shape
    out, av = np.zeros((n, G, D)), np.zeros((n, G, D))
    lse, mass, big = np.full((n, G), -np.inf), np.zeros((n, G)), np.zeros((n, G))
    for i in range(n):
        m = base + i
        vis = np.arange(len(pos)) <= m
        if window:
            vis &= (pos > pos[m] - window) | (pos < n_sink)
        if see is not None:
            vis &= see
        j = np.flatnonzero(vis)
        if not len(j):
            continue
        kk, vv = k[j].astype(np.float64), v[j].astype(np.float64)
        for g in range(G):
            qq = q[i, g].astype(np.float64)
            s = kk @ qq / math.sqrt(D)
            e = np.exp(s - s.max())
            a = e / e.sum()
            out[i, g], av[i, g] = a @ vv, a @ np.abs(vv)
            lse[i, g] = s.max() + math.log(e.sum())
            mass[i, g] = a[pos[j] > pos[m] - suffix_w].sum()
            big[i, g] = (np.abs(kk) @ np.abs(qq)).max() / math.sqrt(D)
    return out, lse, mass, av, big
