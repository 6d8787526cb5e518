"""Drafted tokens: pdn_slot_draft (scores them, applies the accepted ones in the
next call), pdn_draft_verify, and the two in a loop with pdn_slot_fwd.

Bars of the rule: those of the state-pool tests (fp32 arithmetic, one rounding
of o to io).  The verification's outputs are whole numbers: equal."""
import numpy as np
import pytest

from slot_util import KW, batch, dev, dev_batch, host, i32, pool, tokens
from test_gpu_slots import bars, rel_err

pytestmark = pytest.mark.gpu


def tape_of(P, T, H, dk, dv, gate, precond):
    import torch
    import paper_2604_21100_amd as pdn
    # records nobody wrote are never used: NaN would show
    return (torch.full((P, T, H, pdn.pdn_tape_record(dk, dv, gate, precond)), float("nan"), device="cuda"),
            torch.zeros(P, H, dtype=torch.int32, device="cuda"))


CASES = [
    # (io, gate, precond, knorm, H, Hk, dk, dv, most tokens)
    ("bf16", "scalar", "squash", "none", 2, 2, 128, 128, 5),
    ("bf16", "scalar", "identity", "none", 4, 2, 128, 128, 8),
    ("bf16", "channel", "squash", "none", 2, 1, 128, 128, 8),
    ("f32", "none", "squash", "none", 2, 2, 64, 64, 1),
    ("f32", "channel", "identity", "none", 2, 2, 128, 64, 1),
    ("f32", "scalar", "external", "none", 3, 1, 64, 128, 4),
    ("bf16", "channel", "diag_sm", "none", 2, 2, 128, 64, 7),
    ("f32", "scalar", "atq", "none", 2, 2, 128, 128, 6),
    ("bf16", "channel", "atq", "none", 2, 2, 64, 64, 8),
    ("bf16", "scalar", "squash", "beta", 2, 2, 64, 128, 3),
    ("bf16", "scalar", "squash", "none", 2, 2, 128, 128, 12),   # more than a block
    ("f32", "channel", "squash", "1pm", 2, 2, 64, 64, 19),
]


@pytest.mark.parametrize("io,gate,precond,knorm,H,Hk,dk,dv,T", CASES)
def test_rounds(io, gate, precond, knorm, H, Hk, dk, dv, T):
    """Rounds of drafts over sequences that come and go: every slot's state is
    that of its accepted tokens, every o that of the tokens fed after them."""
    import torch
    import paper_2604_21100_amd as pdn
    rng = np.random.default_rng(T * 10 + dk)
    P, N = 5, 3
    S, A = pool(rng, P, H, dk, dv, precond)
    Sd, Ad = dev(S), dev(A)
    tape, pending = tape_of(P, T, H, dk, dv, gate, precond)
    waiting = [None] * P    # the oracle's view: the batch and rows pending in a slot
    bo, bs = bars(io, T)
    worst = [0.0, 0.0, 0.0]
    for rnd in range(6):
        slots = rng.permutation(P)[:N]
        if rnd == 4:
            slots[1] = -1   # padding
        lens = rng.integers(0 if rnd else 1, T + 1, N)
        lens[rnd % N] = T
        if rnd == 5:
            lens[:] = 0     # only the accepted tokens are applied
        starts = np.concatenate([[0], np.cumsum(lens)])
        b = batch(rng, int(starts[-1]), H, Hk, dk, dv, io, gate, precond)
        acc, fresh = rng.integers(-1, T + 3, N), [0, int(rnd == 3), 0]
        pos, opt = dev_batch(b, io, precond, strided=rnd % 2 == 1)
        o = torch.full(b["v"].shape, float("nan"), dtype=pos[0].dtype, device="cuda")
        pdn.pdn_slot_draft(*pos, Sd, tape, pending, accepted=None if rnd == 0 else i32(acc), starts=i32(starts),
                           slots=i32(slots), fresh=i32(fresh), max_tokens=T, A=Ad, gate=gate, precond=precond,
                           knorm=knorm, o=o, **opt, **KW)
        torch.cuda.synchronize()
        ro = np.full(b["v"].shape, np.nan)
        for n, p in enumerate(slots):
            if p < 0:
                continue
            s, a = S[p], None if A is None else A[p]
            if fresh[n]:
                s, a = 0 * s, None if a is None else 0 * a
            elif waiting[p] is not None and rnd:
                old, rows = waiting[p]
                _, s, a = tokens(old, rows[:max(acc[n], 0)], s, a, gate, precond, knorm)
            S[p] = s
            if A is not None:
                A[p] = a
            rows = np.arange(starts[n], starts[n + 1])
            ro[rows] = tokens(b, rows, s, a, gate, precond, knorm)[0]
            waiting[p] = (b, rows)
        got = host(o)
        assert np.array_equal(np.isnan(got), np.isnan(ro))
        live = ~np.isnan(ro)
        errs = (rel_err(got[live], ro[live]), rel_err(host(Sd), S), rel_err(host(Ad), A) if A is not None else 0.0)
        worst = [max(x, y) for x, y in zip(worst, errs)]
        want = [[0 if w is None else len(w[1])] * H for w in waiting]
        assert pending.cpu().tolist() == want
    print(f"{io}/{gate}/{precond} T={T}: o %.2e S %.2e A %.2e" % tuple(worst))
    assert worst[0] <= bo and worst[1] <= bs and worst[2] <= bs, worst


@pytest.mark.parametrize("gate", ["scalar", "channel"])
def test_forked_drafts(gate):
    """A slot's accepted drafts go to two other slots; the slot itself, its tape
    and count stay."""
    import torch
    import paper_2604_21100_amd as pdn
    rng = np.random.default_rng(3)
    H, d, T, P = 2, 128, 6, 4
    S, A = pool(rng, P, H, d, d, "squash")
    Sd, Ad = dev(S), dev(A)
    tape, pending = tape_of(P, T, H, d, d, gate, "squash")
    b = batch(rng, T, H, H, d, d, "bf16", gate, "squash")
    pos, opt = dev_batch(b, "bf16", "squash")
    kw = dict(A=Ad, gate=gate, max_tokens=T, **KW)
    pdn.pdn_slot_draft(*pos, Sd, tape, pending, starts=i32([0, T]), slots=i32([2]), **opt, **kw)
    assert np.array_equal(host(Sd), S)
    kept = tape[2].clone()
    b2 = batch(rng, 5, H, H, d, d, "bf16", gate, "squash")
    pos2, opt2 = dev_batch(b2, "bf16", "squash")
    o = pdn.pdn_slot_draft(*pos2, Sd, tape, pending, accepted=i32([3, 6]), starts=i32([0, 2, 5]), slots=i32([2, 2]),
                           slots_out=i32([0, 3]), **opt2, **kw)
    for n, (dst, acc, lo, hi) in enumerate(((0, 3, 0, 2), (3, 6, 2, 5))):
        _, s, a = tokens(b, np.arange(acc), S[2], A[2], gate, "squash")
        ro = tokens(b2, np.arange(lo, hi), s, a, gate, "squash")[0]
        assert rel_err(host(Sd)[dst], s) <= 1e-5 and rel_err(host(Ad)[dst], a) <= 1e-5
        assert rel_err(host(o)[lo:hi], ro) <= 2 ** -8 + 1e-5
    assert np.array_equal(host(Sd)[[1, 2]], S[[1, 2]]) and torch.equal(tape[2], kept)
    assert pending.cpu().tolist() == [[2, 2], [0, 0], [6, 6], [3, 3]]


@pytest.mark.parametrize("T", [4, 8, 20])
@pytest.mark.parametrize("gate", ["scalar", "channel"])
def test_strong_decay_of_drafts(T, gate):
    """Accepted tokens whose log-decays add up to hundreds, or hold -inf without the
    per-channel gate.  A record has its sum G rounded to fp32, so a decay, the
    exponential of a difference of two, is off by 2 x 2^-24 |G| of itself; at most
    three updates since the last strong decay count, each within the largest value.
    A token's log-decay counts as -128 at the least."""
    import paper_2604_21100_amd as pdn
    rng = np.random.default_rng(31 + T)
    H, d, P = 2, 128, 3
    S, A = pool(rng, P, H, d, d, "squash")
    Sd, Ad = dev(S), dev(A)
    tape, pending = tape_of(P, T, H, d, d, gate, "squash")
    b = batch(rng, P * T, H, H, d, d, "f32", gate, "squash")
    for n in range(P):
        for t in range(0, T, 3):
            b["g"][n * T + t] = [-np.inf, -400.0, -90.0][n] if gate == "scalar" else -25.0
    pos, opt = dev_batch(b, "f32", "squash")
    kw = dict(A=Ad, gate=gate, max_tokens=T, **KW)
    starts = [n * T for n in range(P + 1)]
    o = host(pdn.pdn_slot_draft(*pos, Sd, tape, pending, starts=i32(starts), **opt, **kw))
    acc = [T, T - 1, 2]
    pdn.pdn_slot_draft(*pos, Sd, tape, pending, accepted=i32(acc), starts=i32([0] * (P + 1)), **opt, **kw)
    for n in range(P):
        rows = np.arange(n * T, (n + 1) * T)
        ro = tokens(b, rows, S[n], A[n], gate, "squash")[0]
        _, s, a = tokens(b, rows[:acc[n]], S[n], A[n], gate, "squash")
        G = np.abs(np.maximum(b["g"][rows], -128.0).sum(0)).max()
        e = rel_err(o[rows], ro), rel_err(host(Sd)[n], s), rel_err(host(Ad)[n], a)
        print(gate, T, n, e, G)
        assert e[0] <= 1e-5 and e[1] <= 1e-5 + 3 * 2.0 ** -23 * G and e[2] <= 1e-5


# ------------------------------------------------------------- verification
def ref_verify(p, q, ids, u, r, starts):
    acc, tok = [], []
    V = p.shape[1]
    for n in range(len(starts) - 1):
        lo, hi = starts[n], starts[n + 1]
        if hi <= lo:
            acc.append(0)
            tok.append(-1)
            continue
        row = lo
        while row + 1 < hi:
            x = ids[row + 1]
            if not (0 <= x < V and u[row] * (1.0 if q is None else q[row + 1, x]) < p[row, x]):
                break
            row += 1
        w = np.where(p[row] > 0, p[row], 0.0)
        if row + 1 < hi:
            if q is not None:
                d = p[row] - q[row + 1]
                rest = np.where(d > 0, d, 0.0)
            else:
                rest = w.copy()
                if 0 <= ids[row + 1] < V:
                    rest[ids[row + 1]] = 0.0
            w = rest if rest.sum() > 0 else w
        acc.append(row - lo + 1)
        if not w.sum() > 0:
            tok.append(-1)
            continue
        over = np.nonzero(np.cumsum(w) > r[n] * w.sum())[0]
        tok.append(int(over[0]) if len(over) else int(np.nonzero(w)[0][-1]))
    return acc, tok


def probs(rng, rows, V, dtype):
    import torch
    z = 2.0 * rng.standard_normal((rows, V))
    t = torch.softmax(torch.from_numpy(z), 1).to(dtype).cuda()
    return t, t.double().cpu().numpy()


@pytest.mark.parametrize("V", [1, 7, 512, 2048, 2049, 8193, 24576, 24577, 50257, 300_000])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("given", [True, False])
def test_verify(V, dtype, given):
    import torch
    import paper_2604_21100_amd as pdn
    rng = np.random.default_rng(V + given)
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    lens = [1, 5, 0, 2, 8, 3]
    starts = np.concatenate([[0], np.cumsum(lens)])
    M = int(starts[-1])
    p, P = probs(rng, M, V, dt)
    q, Q = probs(rng, M, V, dt) if given else (None, None)
    if given:   # some drafts from the target itself hold always
        q[5], Q[5] = p[4], P[4]
    ids = np.array([rng.choice(V, p=(Q if given else P)[t] / (Q if given else P)[t].sum()) for t in range(M)])
    if V > 1:
        ids[8] = V    # no such token: does not hold
    u, r = rng.random(M).astype(np.float32), rng.random(len(lens)).astype(np.float32)
    u[:3] = 0.0       # holds wherever p is not zero
    acc, tok = pdn.pdn_draft_verify(p, i32(ids), dev(u), dev(r), q=q, starts=i32(starts))
    wa, wt = ref_verify(P, Q, ids, u.astype(np.float64), r.astype(np.float64), starts)
    print(wa, wt)
    assert acc.cpu().tolist() == wa and tok.cpu().tolist() == wt


def test_verify_long_drafts_and_edges():
    """More drafts than a wave, the ends of r, rows without weight, NaN and
    infinities, residuals that are zero everywhere."""
    import torch
    import paper_2604_21100_amd as pdn
    rng = np.random.default_rng(9)
    V, M = 33, 200
    p, P = probs(rng, M, V, torch.float32)
    ids = rng.integers(0, V, M)
    u = np.zeros(M, dtype=np.float32)     # every draft holds ...
    for stop in (M, 1, 63, 64, 65, 130):  # ... up to this one
        u[:] = 0.0
        if stop < M:
            u[stop - 1] = 1.0
        acc, _ = pdn.pdn_draft_verify(p, i32(ids), dev(u), dev(np.array([0.5])), starts=i32([0, M]))
        assert acc.cpu().tolist() == [min(stop, M)]
    # a row each: ends of r, zeros at the ends, nothing, NaN, infinity
    rows = np.zeros((8, 6), dtype=np.float32)
    rows[:4, 2:4] = 0.5
    rows[5] = np.nan
    rows[6] = [0.25, np.nan, 0.25, 0, 0.5, 0]
    rows[7] = [0, 0.5, np.inf, 0.5, 0, 0]
    r = np.array([0.0, 0.5, 1.0 - 2.0 ** -24, 1.0, 0.3, 0.3, 0.5, 0.3], dtype=np.float32)
    half = np.full((2, 4), 0.25, dtype=np.float32)
    for zeros in (0, 9000, 30_000):   # tokens without a weight around them: every form and segment
        for before in (0, zeros // 2):
            wide = lambda z: dev(np.pad(z, ((0, 0), (before, zeros - before))))   # noqa: E731
            acc, tok = pdn.pdn_draft_verify(wide(rows), i32([0] * 8), dev(np.zeros(8)), dev(r), starts=i32(range(9)))
            assert acc.cpu().tolist() == [1] * 8
            # (an infinite whole: nothing is over the target, so the last token with a weight)
            assert tok.cpu().tolist() == [x if x < 0 else before + x for x in (2, 3, 3, 3, -1, -1, 4, 3)]
            # p under q everywhere: the draft may be refused, the next token is drawn from p
            acc, tok = pdn.pdn_draft_verify(wide(half), i32([0, before + 1]), dev(np.array([1.0, 0.0])),
                                            dev(np.array([0.6])), q=wide(half), starts=i32([0, 2]))
            assert acc.cpu().tolist() == [1] and tok.cpu().tolist() == [before + 2]
    # even rows without starts; starts that leave the tensors
    acc, tok = pdn.pdn_draft_verify(dev(rows), i32([0] * 8), dev(np.ones(8)), dev(r[:4]))
    assert acc.cpu().tolist() == [1] * 4
    acc, tok = pdn.pdn_draft_verify(dev(rows), i32([0] * 8), dev(np.ones(8)), dev(r[:3]), starts=i32([-9, -3, 50, 2]))
    assert acc.cpu().tolist() == [0, 1, 0] and tok.cpu().tolist()[0] == -1


def test_empty_calls():
    import torch
    import paper_2604_21100_amd as pdn
    e = dict(dtype=torch.int32, device="cuda")
    f = lambda *s: torch.empty(*s, device="cuda")   # noqa: E731
    acc, tok = pdn.pdn_draft_verify(f(0, 5), torch.empty(0, **e), f(0), f(0))
    assert acc.numel() == 0
    acc, tok = pdn.pdn_draft_verify(f(0, 5), torch.empty(0, **e), f(0), f(2), starts=torch.zeros(3, **e))
    assert acc.cpu().tolist() == [0, 0] and tok.cpu().tolist() == [-1, -1]
    S = torch.zeros(2, 2, 64, 64, device="cuda")
    o = pdn.pdn_slot_fwd(f(0, 2, 64), f(0, 2, 64), f(0, 2, 64), f(0, 2), S, precond="identity",
                         starts=torch.zeros(3, **e), max_tokens=1)
    assert o.shape == (0, 2, 64) and not S.any()


# ------------------------------------------------- all of it, as a server runs it
@pytest.mark.parametrize("graph", [False, True])
def test_prompt_draft_verify_loop(graph):
    """Prompts into slots, rounds of drafts whose acceptance never leaves the
    device, and the states at the end: those of the tokens that held.  As a
    captured graph of draft and verify too, replayed each round."""
    import torch
    import paper_2604_21100_amd as pdn
    rng = np.random.default_rng(21)
    H, Hk, d, T, N, V = 4, 2, 128, 5, 3, 1000
    S, A = pool(rng, N, H, d, d, "squash")
    Sd, Ad = torch.full((N, H, d, d), float("nan"), device="cuda"), torch.full((N, H, d), float("nan"), device="cuda")
    lens = [40, 3, 17]
    b = batch(rng, sum(lens), H, Hk, d, d, "bf16", "scalar", "squash")
    starts = np.concatenate([[0], np.cumsum(lens)])
    pos, opt = dev_batch(b, "bf16", "squash")
    pdn.pdn_slot_fwd(*pos, Sd, A=Ad, gate="scalar", starts=i32(starts), fresh=i32([1] * N), max_tokens=40, **opt, **KW)
    S, A = np.zeros_like(S), np.zeros_like(A)
    for n in range(N):
        _, S[n], A[n] = tokens(b, np.arange(starts[n], starts[n + 1]), S[n], A[n], "scalar", "squash")
    tape, pending = tape_of(N, T, H, d, d, "scalar", "squash")
    accepted = torch.zeros(N, dtype=torch.int32, device="cuda")
    token = torch.zeros(N, dtype=torch.int32, device="cuda")
    ws = torch.empty(pdn.pdn_draft_verify_workspace_size(N, V), dtype=torch.uint8, device="cuda")
    M = N * T
    bufs, held = None, [None] * N
    for rnd in range(5):
        b = batch(rng, M, H, Hk, d, d, "bf16", "scalar", "squash")
        p, P = probs(rng, M, V, torch.float32)
        q, Q = probs(rng, M, V, torch.float32)
        mix = 0.2 * q + 0.8 * torch.roll(p, 1, 0)
        q, Q = mix, mix.double().cpu().numpy()
        ids = np.array([rng.choice(V, p=Q[t] / Q[t].sum()) for t in range(M)])
        u, r = rng.random(M).astype(np.float32), rng.random(N).astype(np.float32)
        pos, opt = dev_batch(b, "bf16", "squash")
        new = [*pos, opt["g"], opt["beta_p"], opt["g_p"], p, q, i32(ids), dev(u), dev(r)]
        if bufs is None:
            bufs = [x.clone() for x in new]
            o, log_a = torch.empty_like(bufs[2]), opt["log_a_scale"]   # (a graph holds on to no tensor)
            run = lambda: (   # noqa: E731
                pdn.pdn_slot_draft(*bufs[:4], Sd, tape, pending, accepted=accepted, g=bufs[4], gate="scalar",
                                   beta_p=bufs[5], g_p=bufs[6], log_a_scale=log_a, A=Ad, max_tokens=T,
                                   o=o, **KW),
                pdn.pdn_draft_verify(bufs[7], bufs[9], bufs[10], bufs[11], q=bufs[8], accepted=accepted, token=token,
                                     workspace=ws))
            if graph:
                g = torch.cuda.CUDAGraph()
                with torch.cuda.graph(g):   # (captured, not run)
                    run()
        for x, y in zip(bufs, new):
            x.copy_(y)
        g.replay() if graph else run()
        torch.cuda.synchronize()
        wa, wt = ref_verify(P, Q, ids, u.astype(np.float64), r.astype(np.float64), np.arange(N + 1) * T)
        assert accepted.cpu().tolist() == wa and token.cpu().tolist() == wt
        for n in range(N):
            if held[n] is not None:
                old, rows = held[n]
                _, S[n], A[n] = tokens(old, rows, S[n], A[n], "scalar", "squash")
            held[n] = (b, np.arange(n * T, n * T + wa[n]))
            ro = tokens(b, np.arange(n * T, (n + 1) * T), S[n], A[n], "scalar", "squash")[0]
            assert rel_err(host(o)[n * T:(n + 1) * T], ro) <= 2 ** -8 + 3e-5
        assert rel_err(host(Sd), S) <= 3e-5 and rel_err(host(Ad), A) <= 3e-5

