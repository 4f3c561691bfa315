"""What a caller keeps beside the paged cache: the guard's state of sequences that take no step, and of forked ones."""
import numpy as np
import pytest
import torch

from test_paged_step import B, CAP, D, HKV, HQ, L, RING, Paged, _i32, _params, _tokens

pytestmark = pytest.mark.gpu


def _guard(a, tokens, t, idle=None):
    """Steps 4 to 6; the state of idle sequences is put back and their decisions are zeroed."""
    lg = a.lg
    was = a.state.clone()
    lg.lg_detect_loop(a.params, tokens, RING, t, a.zero, a.conf, a.state, a.decision)
    if idle is not None:
        a.state.copy_(torch.where(idle[:, None], was, a.state))
        a.decision.masked_fill_(idle[:, None], 0)
    lg.lg_prune_compact(a.params, B, CAP, [], a.pos, a.len, a.budget, None, a.decision, a.keep, a.new_len)
    lg.lg_page_compact(a.map, a.layers, a.keep, a.new_len, a.moved, a.ws)


def _run(rows, idles, restore=True):
    """130 tokens of every sequence; idles[s] are the sequences that bring none in step s."""
    from paper_2604_10044_amd import lg
    a, tokens, t, seen = Paged(torch.bfloat16, _params(lg)), _tokens(), np.full(B, -1), []
    s = 0
    while t.min() < 129:
        n = np.array([0 if b in idles(s) or t[b] >= 129 else 1 for b in range(B)])
        t, s = t + n, s + 1
        if not n.any():
            continue
        x = torch.stack([rows[b, t[b]] for b in range(B) if n[b]], 1).contiguous()
        a.attend(x, _i32(np.concatenate([[0], np.cumsum(n)])), _i32(t), 1)
        idle = torch.as_tensor(n == 0, device="cuda")
        _guard(a, tokens, _i32(t), idle if restore else None)
        for b in range(B):
            if n[b]:
                seen.append((b, int(t[b]), a.decision[b].tolist()))
    torch.cuda.synchronize()
    live = [a.pos[b, :int(a.len[b])].tolist() for b in range(B)]
    kv = [[a.rows(y[l], b, int(a.len[b])).clone() for l in range(L) for y in (a.k, a.v)] for b in range(B)]
    return sorted(seen), a.state.cpu().numpy(), live, kv


def test_sequences_without_a_token_take_no_step():
    """Sequences that pause come to the decisions, prunes and caches that they have without pauses; a detector step for
    a sequence that pauses, with nothing put back, is one too many."""
    g = torch.Generator(device="cuda").manual_seed(6)
    rows = torch.randn(B, 130, L, HQ + 2 * HKV, D, generator=g, device="cuda").to(torch.bfloat16)
    straight = _run(rows, lambda s: ())
    paused = _run(rows, lambda s: (0,) if s % 3 == 1 else (1, 2) if s % 5 == 2 else ())
    assert straight[0] == paused[0] and straight[2] == paused[2]
    np.testing.assert_array_equal(straight[1], paused[1])
    for x, y in zip(straight[3], paused[3]):
        assert all(torch.equal(u, v) for u, v in zip(x, y))
    assert any(d[0] for _, _, d in straight[0]), "no trigger"
    counted = _run(rows, lambda s: (0,) if s % 3 == 1 else (), restore=False)
    assert [x for x in counted[0] if x[0] == 0] != [x for x in straight[0] if x[0] == 0]


def test_forked_sequences_take_the_guards_rows_along():
    """Copies of a sequence that are fed its tokens, with its row of the state and ring, get its decisions."""
    from paper_2604_10044_amd import lg
    g = torch.Generator(device="cuda").manual_seed(7)
    rows = torch.randn(140, L, 1, HQ + 2 * HKV, D, generator=g, device="cuda").to(torch.bfloat16)
    a, tokens, fired = Paged(torch.bfloat16, _params(lg)), _tokens(), 0
    for t in range(140):
        if t == 70:
            parent = _i32([0, 0, 0])
            lg.lg_page_fork(a.map, parent, a.ws)
            for x in (a.state, tokens, a.budget, a.sw, a.conf):
                x.copy_(x[parent.long()].clone())
        td = _i32([t] * B)
        a.attend(rows[t].expand(L, B, -1, -1).contiguous(), _i32(range(B + 1)), td, 1)
        _guard(a, tokens, td)
        if t >= 70:
            assert a.decision[1].equal(a.decision[0]) and a.decision[2].equal(a.decision[0])
            assert a.state[1].equal(a.state[0]) and a.len[1] == a.len[0] and a.pos[1].equal(a.pos[0])
            fired += int(a.decision[0, 0])
    assert fired
    torch.cuda.synchronize()
    assert int(a.ref.sum()) == int((a.table >= 0).sum())
