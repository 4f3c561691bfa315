"""The paged cache's calls together, as a serving loop makes them: prompts in pieces, then guarded decode steps
with prunes, against the contiguous cache's lg_decode_attend, lg_detect_loop and lg_prune_compact on
the same rows; the step captured as a HIP graph; sequences forked in mid-stream."""
import numpy as np
import pytest
import torch


pytestmark = pytest.mark.gpu

B, L, HQ, HKV, D, PS, P = 3, 2, 8, 2, 64, 16, 8
CAP, BUDGET = PS * P, 96
VOCAB, RING = 1000, 2048


class Paged:
    def __init__(self, dtype, params, n_pages=B * P + 4):
        from paper_2604_10044_amd import lg
        self.lg, self.dtype, self.params = lg, dtype, params
        i32 = lambda *s, v=0: torch.full(s, v, dtype=torch.int32, device="cuda")  # noqa: E731
        self.table, self.pos, self.len, self.ref = i32(B, P, v=-1), i32(B, CAP), i32(B), i32(n_pages)
        self.k = torch.full((L, n_pages, HKV, PS, D), float("nan"), dtype=dtype, device="cuda")  # unwritten rows
        self.v = torch.full_like(self.k, float("nan"))
        self.layers = [lg.paged_layer(self.k[l], self.v[l], HQ) for l in range(L)]
        self.map = lg.page_map(self.table, self.pos, self.len, self.ref, PS)
        self.ws = torch.empty(lg.lg_page_workspace(self.map), dtype=torch.uint8, device="cuda")
        self.ws_attend = torch.empty(lg.lg_paged_attend_workspace(self.layers[0], self.map, B * 64, 64),
                                     dtype=torch.uint8, device="cuda")
        p = lg.RopeParams(lg.LG_ROPE_RAMP, D, 1e4, 4.0, 512.0, 1.0, 32.0)
        freq, self.scale = lg.lg_rope_frequencies(p)
        self.freq = freq.cuda()
        self.base, self.moved, self.new_len = i32(B), i32(B), i32(B)
        self.keep, self.budget, self.zero = i32(B, CAP), i32(B, v=BUDGET), i32(B)
        self.sw = i32(B, v=BUDGET // 4)
        self.state = torch.zeros(B, lg.STATE_INTS, dtype=torch.int32, device="cuda")
        self.decision = torch.zeros(B, lg.DECISION_INTS, dtype=torch.int32, device="cuda")
        self.conf = torch.zeros(B, device="cuda")

    def attend(self, qkv, q_start, t, chunk):
        """qkv [L][T][HQ + 2 HKV][D]; returns rotated queries, outputs, lse and suffix masses of the layers."""
        lg, T = self.lg, qkv.shape[1]
        lg.lg_page_reserve(self.map, self.layers, q_start, t, self.base, self.ws)
        got = []
        for l in range(L):
            q = torch.zeros(T, HQ, D, dtype=self.dtype, device="cuda")
            out, lse, sm = torch.zeros_like(q), torch.zeros(T, HQ, device="cuda"), torch.zeros(T, HQ, device="cuda")
            lg.lg_rope_append(self.layers[l], self.map, qkv[l, :, :HQ], qkv[l, :, HQ:HQ + HKV], qkv[l, :, HQ + HKV:],
                              self.freq, D, False, self.scale, q, q_start, self.base)
            lg.lg_paged_attend(self.layers[l], self.map, q, out, q_start, self.base, chunk, 0, 0, self.sw, lse, sm,
                               self.conf, self.ws_attend)
            got.append((q, out, lse, sm))
        return got

    def guard(self, tokens, t):
        lg = self.lg
        lg.lg_detect_loop(self.params, tokens, RING, t, self.zero, self.conf, self.state, self.decision)
        lg.lg_prune_compact(self.params, B, CAP, [], self.pos, self.len, self.budget, None, self.decision, self.keep,
                            self.new_len)
        lg.lg_page_compact(self.map, self.layers, self.keep, self.new_len, self.moved, self.ws)

    def rows(self, x, b, n):
        """Rows of sequence b's first n slots, [HKV][n][D]."""
        page = self.table[b, torch.arange(n, device="cuda") // PS].long()
        return x[page, :, torch.arange(n, device="cuda") % PS].transpose(0, 1)


def _tokens():
    """Loops of periods 5 and 9 from position 60 on in two sequences, the third without one."""
    r = np.random.RandomState(0)
    y = r.randint(0, VOCAB, (B, RING)).astype(np.int32)
    for b, p in ((0, 5), (2, 9)):
        y[b, 60:] = np.resize(r.randint(0, VOCAB, p), RING - 60)
    return torch.as_tensor(y, device="cuda")


def _params(lg):
    return lg.params_from_dict(dict(W=64, n_anchor=4, t_min=32))


def _i32(x):
    return torch.as_tensor(np.asarray(x, np.int32), device="cuda")


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_guarded_loop_matches_the_contiguous_cache(dtype):
    from paper_2604_10044_amd import lg
    params = _params(lg)
    a = Paged(dtype, params)
    g = torch.Generator(device="cuda").manual_seed(1)
    rand = lambda T: torch.randn(L, T, HQ + 2 * HKV, D, generator=g, device="cuda").to(dtype)  # noqa: E731
    tokens = _tokens()
    # prompts of 50, 20 and 33 tokens in two pieces
    t = np.full(B, -1)
    for n in ([30, 20, 1], [20, 0, 32]):
        t = t + n
        a.attend(rand(sum(n)), _i32(np.concatenate([[0], np.cumsum(n)])), _i32(t), max(n))
    a.conf.zero_()
    # the contiguous cache takes over the same rows
    K = [torch.zeros(B, HKV, CAP, D, dtype=dtype, device="cuda") for _ in range(L)]
    V = [torch.zeros_like(K[0]) for _ in range(L)]
    pos, ln = a.pos.clone(), a.len.clone()
    for b in range(B):
        n = int(ln[b])
        for l in range(L):
            K[l][b, :, :n], V[l][b, :, :n] = a.rows(a.k[l], b, n), a.rows(a.v[l], b, n)
    acc = [torch.zeros(B, HKV, CAP, device="cuda") for _ in range(L)]
    flat = [lg.layer_cache(K[l], V[l], acc[l], HQ) for l in range(L)]
    ws = torch.empty(lg.lg_decode_attend_workspace(flat[0]), dtype=torch.uint8, device="cuda")
    lg.lg_decode_attend_workspace_init(flat[0], ws)
    state, decision = torch.zeros_like(a.state), torch.zeros_like(a.decision)
    conf, keep, new_len = torch.zeros_like(a.conf), torch.zeros_like(a.keep), torch.zeros_like(a.new_len)
    q_start = _i32(range(B + 1))
    prunes = 0
    for step in range(120):
        t = t + 1
        td = _i32(t)
        qkv = rand(B)
        got = a.attend(qkv, q_start, td, 1)
        slot = a.base.cpu().numpy()
        np.testing.assert_array_equal(slot, ln.cpu().numpy())
        for l in range(L):
            q, out, lse, sm = got[l]
            kn = torch.stack([a.rows(a.k[l], b, slot[b] + 1)[:, -1] for b in range(B)]).contiguous()
            vn = torch.stack([a.rows(a.v[l], b, slot[b] + 1)[:, -1] for b in range(B)]).contiguous()
            assert torch.equal(vn, qkv[l, :, HQ + HKV:])
            o, ls, s = torch.zeros_like(out), torch.zeros_like(lse), torch.zeros_like(sm)
            lg.lg_decode_attend(flat[l], q, kn, vn, o, pos, ln, td, a.sw, ls, s, conf, ws)
            # two roundings to bfloat16 and the weights'; both within 1e-5 in float32 (sums of 100 terms)
            tol = 3 * 2.0 ** -8 * 4.5 if dtype is torch.bfloat16 else 1e-5
            assert (out.float() - o.float()).abs().max() <= tol
            assert (lse - ls).abs().max() <= 1e-5 and (sm - s).abs().max() <= 1e-5
        a.guard(tokens, td)
        lg.lg_detect_loop(params, tokens, RING, td, a.zero, conf, state, decision)
        lg.lg_prune_compact(params, B, CAP, flat, pos, ln, a.budget, td, decision, keep, new_len)
        torch.cuda.synchronize()
        for x, y in ((a.decision, decision), (a.len, ln), (a.new_len, new_len)):
            np.testing.assert_array_equal(x.cpu().numpy(), y.cpu().numpy(), err_msg="step %d" % step)
        assert (a.moved.cpu().numpy() == (new_len.cpu().numpy() >= 0)).all()
        prunes += int((new_len >= 0).sum())
        for b in range(B):
            n = int(ln[b])
            np.testing.assert_array_equal(a.pos[b, :n].cpu().numpy(), pos[b, :n].cpu().numpy())
            assert int((a.table[b] >= 0).sum()) == -(-n // PS)
            for l in range(L):
                assert torch.equal(a.rows(a.k[l], b, n), K[l][b, :, :n]) and torch.equal(a.rows(a.v[l], b, n), V[l][b, :, :n])
        assert int(a.ref.sum()) == int((a.table >= 0).sum())
    assert prunes >= 4
    assert bool(a.decision[:, 13].max() >= 1), "no intervention"


def test_step_graph_replay_matches_eager():
    """The whole step in one graph, replayed with eager work and synchronisations between the replays."""
    from paper_2604_10044_amd import lg
    tokens = _tokens()
    g = torch.Generator(device="cuda").manual_seed(2)
    steps, first = 40, 70
    prompt = torch.randn(L, B * first, HQ + 2 * HKV, D, generator=g, device="cuda").to(torch.bfloat16)
    rows = torch.randn(steps, L, B, HQ + 2 * HKV, D, generator=g, device="cuda").to(torch.bfloat16)
    chunk = _i32([0, first, 2 * first, 3 * first])
    q_start = _i32(range(B + 1))

    def start():
        a = Paged(torch.bfloat16, _params(lg))
        a.ws_attend = torch.empty(lg.lg_paged_attend_workspace(a.layers[0], a.map, B * first, first), dtype=torch.uint8,
                                  device="cuda")
        a.attend(prompt, chunk, _i32([first - 1] * B), first)
        a.conf.zero_()
        return a

    def look(a, got):
        torch.cuda.synchronize()
        return [x.float().cpu().numpy().copy() for x in (a.table, a.pos, a.len, a.ref, a.decision, a.new_len, a.moved)] + \
            [x.float().nan_to_num(7.5).cpu().numpy() for x in (a.k, a.v)] + \
            [x.float().cpu().numpy() for r in got for x in r]

    a, want = start(), []
    for s in range(steps):
        t = _i32([first + s] * B)
        got = a.attend(rows[s], q_start, t, 1)
        a.guard(tokens, t)
        want.append(look(a, got))
    a = start()
    t, x = _i32([0] * B), torch.zeros_like(rows[0])
    bufs = [a.table, a.pos, a.len, a.ref, a.state, a.decision, a.conf, a.k, a.v]
    keep = [b.clone() for b in bufs]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = a.attend(x, q_start, t, 1)
        a.guard(tokens, t)
    for b, v in zip(bufs, keep):
        b.copy_(v)
    for s in range(steps):
        t.fill_(first + s)
        x.copy_(rows[s])
        graph.replay()
        for u, w in zip(want[s], look(a, got)):
            np.testing.assert_array_equal(u, w, err_msg="step %d" % s)
        torch.randn(1 << 16, device="cuda").sum()
        torch.cuda.synchronize()


def test_two_graphs_share_a_workspace():
    """Two captured attention calls of different shapes on one workspace, replayed in turn."""
    from paper_2604_10044_amd import lg
    g = torch.Generator(device="cuda").manual_seed(3)
    calls = []
    ws = torch.empty(16 << 20, dtype=torch.uint8, device="cuda")
    for hq, hkv, n in ((4, 2, 1), (8, 1, 9)):
        k, v = (torch.randn(80, hkv, 16, 64, generator=g, device="cuda").to(torch.bfloat16) for _ in range(2))
        table = torch.arange(64, dtype=torch.int32, device="cuda")[None].contiguous()
        pos = torch.arange(1024, dtype=torch.int32, device="cuda")[None].contiguous()
        m = lg.page_map(table, pos, _i32([1000]), torch.ones(80, dtype=torch.int32, device="cuda"), 16)
        q = torch.randn(n, hq, 64, generator=g, device="cuda").to(torch.bfloat16)
        out, lse = torch.zeros_like(q), torch.zeros(n, hq, device="cuda")
        args = (lg.paged_layer(k, v, hq), m, q, out, _i32([0, n]), _i32([1000 - n]), n, 0, 0, None, lse, None, None, ws)
        assert 16 < lg.lg_paged_attend_workspace(args[0], m, n, n) <= ws.numel()
        lg.lg_paged_attend(*args)
        torch.cuda.synchronize()
        want = (out.clone(), lse.clone())
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            lg.lg_paged_attend(*args)
        calls.append((graph, out, lse, want, args))
    for rep in range(4):
        for graph, out, lse, want, _ in calls:
            out.zero_(), lse.zero_()
            graph.replay()
        torch.cuda.synchronize()
        for graph, out, lse, want, _ in calls:
            assert torch.equal(out, want[0]) and torch.equal(lse, want[1])


def test_forked_sequences_part_and_agree():
    """Samples of one prompt: forked sequences that are fed the same tokens stay bit for bit the same, and differ
    from where their tokens do; the parent is not touched by what its copies do."""
    from paper_2604_10044_amd import lg
    a = Paged(torch.bfloat16, _params(lg))
    g = torch.Generator(device="cuda").manual_seed(4)
    rand = lambda T: torch.randn(L, T, HQ + 2 * HKV, D, generator=g, device="cuda").to(torch.bfloat16)  # noqa: E731
    a.attend(rand(37), _i32([0, 37, 37, 37]), _i32([36, -1, -1]), 37)
    lg.lg_page_fork(a.map, _i32([0, 0, 0]), a.ws)
    assert a.table[1].equal(a.table[0]) and a.len.tolist() == [37] * 3
    for s in range(20):
        x = rand(B)
        x[:, 1] = x[:, 0]
        got = a.attend(x, _i32(range(B + 1)), _i32([37 + s] * B), 1)
        for q, out, lse, sm in got:
            assert torch.equal(out[0], out[1]) and torch.equal(lse[0], lse[1]) and not torch.equal(out[0], out[2])
    torch.cuda.synchronize()
    t = a.table.cpu().numpy()
    assert (t[0, :2] == t[1, :2]).all() and (t[0, :2] == t[2, :2]).all()  # whole pages of the prompt stay shared
    assert len({int(x) for x in t[:, 2]}) == 3
    assert a.ref[torch.as_tensor(t[0, :2], device="cuda").long()].tolist() == [3, 3]
    lg.lg_page_fork(a.map, _i32([-1, -1, -1]), a.ws)
    torch.cuda.synchronize()
    assert int(a.ref.abs().sum()) == 0 and a.len.tolist() == [0, 0, 0]


def test_out_of_pages_marks_the_sequence():
    """A sequence that gets no page is refused: its conf is NaN, the detector reports attend_error and its
    cache stays; once another ends, its token is taken."""
    from paper_2604_10044_amd import lg
    a = Paged(torch.bfloat16, _params(lg), n_pages=5)
    g = torch.Generator(device="cuda").manual_seed(5)
    rand = lambda T: torch.randn(L, T, HQ + 2 * HKV, D, generator=g, device="cuda").to(torch.bfloat16)  # noqa: E731
    a.attend(rand(64), _i32([0, 32, 64, 64]), _i32([31, 31, -1]), 32)
    a.conf.zero_()
    tokens = _tokens()
    a.attend(rand(3), _i32(range(B + 1)), _i32([32, 32, 0]), 1)
    assert a.base.tolist() == [32, -1, -1] and a.len.tolist() == [33, 32, 0]
    a.guard(tokens, _i32([32, 32, 0]))
    assert a.decision[:, lg.ATTEND_ERROR_COL].tolist() == [0, 1, 1]
    lg.lg_page_fork(a.map, _i32([-1, 1, 2]), a.ws)
    a.attend(rand(3), _i32(range(B + 1)), _i32([0, 32, 0]), 1)
    assert a.base.tolist() == [0, 32, 0]
    a.guard(tokens, _i32([0, 32, 0]))
    assert a.decision[:, lg.ATTEND_ERROR_COL].tolist() == [0, 0, 0]
