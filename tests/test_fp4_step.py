"""The calls on 4-bit pages together, as a serving loop makes them: prompts in pieces with three axes, then guarded decode
steps with prunes, against the same loop on pages that hold the read-back values; the step as a HIP graph; forks."""
import numpy as np
import pytest
import torch

from oracle import paged

pytestmark = pytest.mark.gpu

B, L, HQ, HKV, D, PS, P = 3, 2, 8, 2, 64, 16, 8
CAP, BUDGET = PS * P, 96
VOCAB, RING = 1000, 2048
SECTIONS = [8, 12, 12]


def _i32(x):
    return torch.as_tensor(np.asarray(x, np.int32), device="cuda")


def _tokens():
    """Loops of periods 5 and 9 from position 60 on in two sequences, the third without one."""
    r = np.random.RandomState(0)
    y = r.randint(0, VOCAB, (B, RING)).astype(np.int32)
    for b, p in ((0, 5), (2, 9)):
        y[b, 60:] = np.resize(r.randint(0, VOCAB, p), RING - 60)
    return torch.as_tensor(y, device="cuda")


class Loop:
    """A paged cache with what a guarded loop keeps beside it; fp4: in 4 bits."""

    def __init__(self, dtype, fp4, n_pages=B * P + 4):
        from paper_2604_10044_amd import lg
        self.lg, self.dtype, self.fp4 = lg, dtype, fp4
        i32 = lambda *s, v=0: torch.full(s, v, dtype=torch.int32, device="cuda")  # noqa: E731
        self.table, self.pos, self.len, self.ref = i32(B, P, v=-1), i32(B, CAP), i32(B), i32(n_pages)
        if fp4:  # unwritten rows stand for NaN
            self.k = torch.full((L, n_pages, HKV, lg.fp4_page_bytes(PS, D)), 255, dtype=torch.uint8, device="cuda")
            self.v = self.k.clone()
            self.layers = [lg.paged_layer_fp4(self.k[l], self.v[l], HQ, PS, D) for l in range(L)]
        else:
            self.k = torch.full((L, n_pages, HKV, PS, D), float("nan"), dtype=dtype, device="cuda")
            self.v = self.k.clone()
            self.layers = [lg.paged_layer(self.k[l], self.v[l], HQ) for l in range(L)]
        self.map = lg.page_map(self.table, self.pos, self.len, self.ref, PS)
        self.ws = torch.empty(lg.lg_page_workspace(self.map), dtype=torch.uint8, device="cuda")
        size = lg.lg_paged_attend_fp4_workspace(self.layers[0], self.map, dtype, B * 80, 80) if fp4 else \
            lg.lg_paged_attend_workspace(self.layers[0], self.map, B * 80, 80)
        self.ws_attend = torch.empty(size, dtype=torch.uint8, device="cuda")
        freq, self.scale = lg.lg_rope_frequencies(lg.RopeParams(lg.LG_ROPE_RAMP, D, 1e4, 4.0, 512.0, 1.0, 32.0))
        self.freq, self.axis = freq.cuda(), lg.lg_rope_axes(SECTIONS, lg.LG_AXES_TURNS).cuda()
        self.base, self.moved, self.new_len, self.zero = i32(B), i32(B), i32(B), i32(B)
        self.keep, self.budget, self.sw = i32(B, CAP), i32(B, v=BUDGET), i32(B, v=BUDGET // 4)
        self.state = torch.zeros(B, lg.STATE_INTS, dtype=torch.int32, device="cuda")
        self.decision = torch.zeros(B, lg.DECISION_INTS, dtype=torch.int32, device="cuda")
        self.conf = torch.zeros(B, device="cuda")
        self.params = lg.params_from_dict(dict(W=64, n_anchor=4, t_min=32))

    def reserve(self, q_start, t):
        self.lg.lg_page_reserve(self.map, self.layers, q_start, t, self.base, self.ws)

    def append(self, l, qkv, coord, q_start):
        q = torch.zeros(len(qkv), HQ, D, dtype=self.dtype, device="cuda")
        self.lg.lg_rope_append_axes(self.layers[l], self.map, qkv[:, :HQ], qkv[:, HQ:HQ + HKV], qkv[:, HQ + HKV:], self.freq, D, False,
                                    self.scale, self.axis, coord, q, q_start, self.base)
        return q

    def attend(self, l, q, q_start, chunk):
        out, lse, sm = torch.zeros_like(q), torch.zeros(len(q), HQ, device="cuda"), torch.zeros(len(q), HQ, device="cuda")
        call = self.lg.lg_paged_attend_fp4 if self.fp4 else self.lg.lg_paged_attend
        call(self.layers[l], self.map, q, out, q_start, self.base, chunk, 0, 0, self.sw, lse, sm, self.conf, self.ws_attend)
        return out, lse, sm

    def step(self, qkv, coord, q_start, t, chunk):
        self.reserve(q_start, t)
        got = []
        for l in range(L):
            q = self.append(l, qkv[l], coord, q_start)
            got.append((q,) + self.attend(l, q, q_start, chunk))
        return got

    def guard(self, tokens, t):
        lg = self.lg
        lg.lg_detect_loop(self.params, tokens, RING, t, self.zero, self.conf, self.state, self.decision)
        lg.lg_prune_compact(self.params, B, CAP, [], self.pos, self.len, self.budget, None, self.decision, self.keep, self.new_len)
        lg.lg_page_compact(self.map, self.layers, self.keep, self.new_len, self.moved, self.ws)

    def read(self, l, n):
        """Values of the first n[b] slots of all sequences, [sum n][HKV][D] twice."""
        start = _i32(np.concatenate([[0], np.cumsum(n)]))
        k, v = (torch.zeros(int(sum(n)), HKV, D, dtype=self.dtype, device="cuda") for _ in range(2))
        self.lg.lg_page_unpack_fp4(self.layers[l], self.map, k, v, start, self.zero)
        return k, v


def _coord(r, t, n):
    """Three axes of the tokens of a step: the newest token of sequence b at t[b] in time, anywhere in height and width."""
    time = np.concatenate([t[b] - n[b] + 1 + np.arange(n[b]) for b in range(B)])
    return _i32(np.stack([time, r.randint(0, 40, len(time)), r.randint(0, 60, len(time))]))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_guarded_loop_matches_pages_of_the_values(dtype):
    """Two loops, one on 4-bit pages and one on pages of the values that these stand for: the same decisions, prunes and
    rows, and outputs within the roundings of both."""
    a, c = Loop(dtype, True), Loop(dtype, False)
    r = np.random.RandomState(1)
    g = torch.Generator(device="cuda").manual_seed(1)
    tokens, t, prunes = _tokens(), np.full(B, -1), 0
    pieces = [[30, 20, 1], [20, 0, 32]] + [[1, 1, 1]] * 120
    for step, n in enumerate(pieces):
        t = t + n
        td, q_start = _i32(t), _i32(np.concatenate([[0], np.cumsum(n)]))
        qkv = torch.randn(L, sum(n), HQ + 2 * HKV, D, generator=g, device="cuda").to(dtype)
        coord = _coord(r, t, n)
        a.reserve(q_start, td)
        c.reserve(q_start, td)
        seq, at = np.repeat(np.arange(B), n), np.concatenate([np.arange(x) for x in n])
        slot = a.base.cpu().numpy()[seq] + at
        for l in range(L):
            q = a.append(l, qkv[l], coord, q_start)
            # the values go to the other cache's rows
            k, v = (torch.zeros(sum(n), HKV, D, dtype=dtype, device="cuda") for _ in range(2))
            a.lg.lg_page_unpack_fp4(a.layers[l], a.map, k, v, q_start, a.base)
            page = c.table.cpu().numpy()[seq, slot // PS]
            c.k[l][page, :, slot % PS], c.v[l][page, :, slot % PS] = k, v
            for (x, ls, s), (y, ls2, s2) in [(a.attend(l, q, q_start, max(n)), c.attend(l, q, q_start, max(n)))]:
                # each weight's rounding and both outputs'; 1e-5 for float32 sums of 100 terms
                tol = 3 * 2.0 ** -8 * float(v.float().abs().max().clamp_min(8)) if dtype is torch.bfloat16 else 2e-5
                assert (x.float() - y.float()).abs().max() <= tol and (ls - ls2).abs().max() <= 1e-5 and (s - s2).abs().max() <= 1e-5
        if step < 2:
            a.conf.zero_(), c.conf.zero_()
            continue
        a.guard(tokens, td)
        c.guard(tokens, td)
        torch.cuda.synchronize()
        for x, y in ((a.decision, c.decision), (a.len, c.len), (a.new_len, c.new_len), (a.table, c.table), (a.ref, c.ref), (a.moved, c.moved)):
            np.testing.assert_array_equal(x.cpu().numpy(), y.cpu().numpy(), err_msg="step %d" % step)
        prunes += int((a.new_len >= 0).sum())
        ln = a.len.cpu().numpy()
        for l in range(L):
            k, v = a.read(l, ln)
            seq, slot = np.repeat(np.arange(B), ln), np.concatenate([np.arange(x) for x in ln])
            page = c.table.cpu().numpy()[seq, slot // PS]
            assert torch.equal(k, c.k[l][page, :, slot % PS]) and torch.equal(v, c.v[l][page, :, slot % PS])
    assert prunes >= 4 and bool(a.decision[:, 13].max() >= 1)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_step_graph_replay_matches_eager(dtype):
    """The whole step in one graph, replayed with eager work and synchronisations between the replays."""
    tokens, steps, first = _tokens(), 30, 70
    g = torch.Generator(device="cuda").manual_seed(2)
    prompt = torch.randn(L, B * first, HQ + 2 * HKV, D, generator=g, device="cuda").to(dtype)
    rows = torch.randn(steps, L, B, HQ + 2 * HKV, D, generator=g, device="cuda").to(dtype)
    coords = [_coord(np.random.RandomState(s), np.full(B, first + s), [1] * B) for s in range(steps)]
    q_start = _i32(range(B + 1))

    def start():
        a = Loop(dtype, True)
        a.step(prompt, _coord(np.random.RandomState(99), np.full(B, first - 1), [first] * B), _i32([0, first, 2 * first, 3 * first]),
               _i32([first - 1] * B), first)
        a.conf.zero_()
        return a

    def look(a, got):
        torch.cuda.synchronize()
        return [x.cpu().numpy().copy() for x in (a.table, a.pos, a.len, a.ref, a.decision, a.new_len, a.moved, a.k, a.v)] + \
            [x.float().cpu().numpy() for y in got for x in y]

    a, want = start(), []
    for s in range(steps):
        t = _i32([first + s] * B)
        got = a.step(rows[s], coords[s], q_start, t, 1)
        a.guard(tokens, t)
        want.append(look(a, got))
    a = start()
    t, x, coord = _i32([0] * B), torch.zeros_like(rows[0]), torch.zeros_like(coords[0])
    bufs = [a.table, a.pos, a.len, a.ref, a.state, a.decision, a.conf, a.k, a.v]
    keep = [b.clone() for b in bufs]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = a.step(x, coord, q_start, t, 1)
        a.guard(tokens, t)
    for b, v in zip(bufs, keep):
        b.copy_(v)
    for s in range(steps):
        t.fill_(first + s)
        x.copy_(rows[s])
        coord.copy_(coords[s])
        graph.replay()
        for u, w in zip(want[s], look(a, got)):
            np.testing.assert_array_equal(u, w, err_msg="step %d" % s)
        torch.randn(1 << 16, device="cuda").sum()
        torch.cuda.synchronize()


def test_two_graphs_share_a_workspace():
    """Two captured attention calls of different shapes and types on one workspace, replayed in turn."""
    from paper_2604_10044_amd import lg
    g = torch.Generator(device="cuda").manual_seed(3)
    calls = []
    ws = torch.empty(32 << 20, dtype=torch.uint8, device="cuda")
    for hq, hkv, n, dtype in ((4, 2, 1, torch.bfloat16), (8, 1, 9, torch.float32)):
        k, v = (torch.randint(0, 256, (80, hkv, lg.fp4_page_bytes(16, 64)), generator=g, device="cuda", dtype=torch.uint8) for _ in range(2))
        k[..., 512:], v[..., 512:] = 127, 126
        table = torch.arange(64, dtype=torch.int32, device="cuda")[None].contiguous()
        pos = torch.arange(1024, dtype=torch.int32, device="cuda")[None].contiguous()
        m = lg.page_map(table, pos, _i32([1000]), torch.ones(80, dtype=torch.int32, device="cuda"), 16)
        q = torch.randn(n, hq, 64, generator=g, device="cuda").to(dtype)
        out, lse = torch.zeros_like(q), torch.zeros(n, hq, device="cuda")
        args = (lg.paged_layer_fp4(k, v, hq, 16, 64), m, q, out, _i32([0, n]), _i32([1000 - n]), n, 0, 0, None, lse, None, None, ws)
        assert lg.lg_paged_attend_fp4_workspace(args[0], m, dtype, n, n) <= ws.numel()
        lg.lg_paged_attend_fp4(*args)
        torch.cuda.synchronize()
        want = (out.clone(), lse.clone())
        assert bool(want[0].isfinite().all())
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            lg.lg_paged_attend_fp4(*args)
        calls.append((graph, out, lse, want, args))
    for rep in range(4):
        for graph, out, lse, want, _ in calls:
            out.zero_(), lse.zero_()
            graph.replay()
        torch.cuda.synchronize()
        for graph, out, lse, want, _ in calls:
            assert torch.equal(out, want[0]) and torch.equal(lse, want[1])


def test_forked_sequences_part_and_agree():
    """Forked sequences that are fed the same tokens stay bit for bit the same and differ from where their tokens do."""
    a = Loop(torch.bfloat16, True)
    g = torch.Generator(device="cuda").manual_seed(4)
    r = np.random.RandomState(4)
    rand = lambda T: torch.randn(L, T, HQ + 2 * HKV, D, generator=g, device="cuda").to(torch.bfloat16)  # noqa: E731
    a.step(rand(37), _coord(r, np.array([36, -1, -1]), [37, 0, 0]), _i32([0, 37, 37, 37]), _i32([36, -1, -1]), 37)
    a.lg.lg_page_fork(a.map, _i32([0, 0, 0]), a.ws)
    for s in range(20):
        x, coord = rand(B), _coord(r, np.full(B, 37 + s), [1] * B)
        x[:, 1], coord[:, 1] = x[:, 0], coord[:, 0]
        for q, out, lse, sm in a.step(x, coord, _i32(range(B + 1)), _i32([37 + s] * B), 1):
            assert torch.equal(out[0], out[1]) and torch.equal(lse[0], lse[1]) and not torch.equal(out[0], out[2])
    k, v = a.read(0, [57] * 3)
    assert torch.equal(k[:57], k[57:114]) and torch.equal(k[:37], k[114:151]) and not torch.equal(k[:57], k[114:])
    assert torch.equal(v[:57], v[57:114])


def test_out_of_pages_marks_the_sequence():
    """A sequence that gets no page is refused: its conf is NaN, the detector reports it, and its cache stays."""
    a = Loop(torch.bfloat16, True, n_pages=5)
    g = torch.Generator(device="cuda").manual_seed(5)
    r = np.random.RandomState(5)
    rand = lambda T: torch.randn(L, T, HQ + 2 * HKV, D, generator=g, device="cuda").to(torch.bfloat16)  # noqa: E731
    a.step(rand(64), _coord(r, np.array([31, 31, -1]), [32, 32, 0]), _i32([0, 32, 64, 64]), _i32([31, 31, -1]), 32)
    a.conf.zero_()
    before = a.read(0, [0, 32, 0])[0]
    a.step(rand(3), _coord(r, np.array([32, 32, 0]), [1] * 3), _i32(range(B + 1)), _i32([32, 32, 0]), 1)
    assert a.base.tolist() == [32, -1, -1] and a.len.tolist() == [33, 32, 0]
    a.guard(_tokens(), _i32([32, 32, 0]))
    assert a.decision[:, a.lg.ATTEND_ERROR_COL].tolist() == [0, 1, 1]
    assert torch.equal(before, a.read(0, [0, 32, 0])[0])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_guarded_loop_rows_against_64_bits(dtype):
    """Every row of a guarded loop's steps against attention in 64 bits on what its pages hold: chunks of prompts, then decode
    steps between prunes. The bounds are those of test_parity_fp4_attend.py: of each weight (2^-8 in bfloat16 chunks, 2^-16 in steps
    of few rows, 0 in float32) times sum alpha |v|, half a step of the result, and float32 sums."""
    a, G = Loop(dtype, True), HQ // HKV
    r = np.random.RandomState(5)
    g = torch.Generator(device="cuda").manual_seed(5)
    tokens, t, prunes, most = _tokens(), np.full(B, -1), 0, 0.0
    for step, n in enumerate([[30, 20, 1], [20, 0, 32]] + [[1, 1, 1]] * 90):
        t = t + n
        q_start = np.concatenate([[0], np.cumsum(n)])
        got = a.step(torch.randn(L, sum(n), HQ + 2 * HKV, D, generator=g, device="cuda").to(dtype), _coord(r, t, n), _i32(q_start), _i32(t), max(n))
        if step < 2 or step % 9 == 0:
            base, pos, sw = (x.cpu().numpy() for x in (a.base, a.pos, a.sw))
            full = base + n
            at = np.concatenate([[0], np.cumsum(full)])
            for l, (q, out, lse, sm) in enumerate(got):
                k, v = (x.double().cpu().numpy() for x in a.read(l, full))
                q, out, lse, sm = (x.double().cpu().numpy() for x in (q, out, lse, sm))
                for b in range(B):
                    if n[b] == 0:
                        continue
                    rows, slots = slice(q_start[b], q_start[b + 1]), slice(at[b], at[b + 1])
                    for h in range(HKV):
                        heads = slice(h * G, (h + 1) * G)
                        o, ls, ms, av, big = paged.attend(q[rows, heads], k[slots, h], v[slots, h], pos[b, :full[b]], base[b], 0, 0, int(sw[b]))
                        err = ((D + 8) * big + 4 * full[b] / 32 + 144) * 2.0 ** -24
                        half, w = (2.0 ** -8, 2.0 ** -8 if n[b] * G > 32 else 2.0 ** -16) if dtype is torch.bfloat16 else (2.0 ** -24, 0.0)
                        tol = (2 * err[..., None] + w) * av * (1 + half) + half * np.abs(o) + full[b] * 2.0 ** -124 * np.abs(v).max()
                        most = max(most, float((tol.max(-1) / av.max(-1)).max()))
                        what = (step, l, b, h)
                        assert (np.abs(out[rows, heads] - o) <= tol).all(), what
                        assert (np.abs(lse[rows, heads] - ls) <= err + 2.0 ** -22 * (np.abs(ls) + big)).all(), what
                        assert (np.abs(sm[rows, heads] - ms) <= 2 * err * ms + full[b] * 2.0 ** -126).all(), what
        if step < 2:
            a.conf.zero_()
            continue
        a.guard(tokens, _i32(t))
        torch.cuda.synchronize()
        prunes += int((a.new_len >= 0).sum())
    assert prunes >= 4 and most < 2.0 ** -6  # beside the row's largest sum alpha |v|: a value too many or too few would show
