"""pdn_slot_fwd: ragged batches of sequences on a pool of states, against the
oracle's token recurrence, sequence by sequence.

Bars.  Arithmetic is fp32 throughout.  A product with the state sums d_k terms:
its error is at most d_k 2^-24 of the terms' magnitudes, 7.6e-6 at 128, and the
write keys' logarithm and exponentials add a few 2^-22; the rule contracts
towards its inputs, so a run does not add up over tokens.  So 1e-5 of the largest
value for a few tokens, and 3e-5 for hundreds, where the largest of some ten
thousand values is taken and a correction is a difference of larger ones.
Outputs are rounded to io once more: bf16 2^-8 of the value.
A value under fp32's smallest normal number, 2^-126, may come out as zero: where a
state has decayed to 1e-75 the oracle has that and fp32 nothing, so errors are
taken of the largest value or of 2^-126 / 1e-5, whichever is more."""
import numpy as np
import pytest

from slot_util import KW, batch, dev, dev_batch, host, i32, pool, tokens

pytestmark = pytest.mark.gpu


def bars(io, T):
    s = 1e-5 if T <= 8 else 3e-5
    return (2 ** -8 + s if io == "bf16" else s), s


def rel_err(x, r):
    """max |x - r| of max |r|, or of what makes 2^-126 an error of 1e-5 (above)."""
    return float(np.abs(x - r).max() / max(np.abs(r).max(), 2.0 ** -126 / 1e-5)) if r.size else 0.0


def run(b, S, A, io, gate, precond, strided=False, knorm="none", **kw):
    """The call on copies of the pool: o (NaN where the call wrote nothing), S, A."""
    import torch
    import paper_2604_21100_amd as pdn
    pos, opt = dev_batch(b, io, precond, strided)
    Sd, Ad = dev(S), dev(A)
    o = torch.full(b["v"].shape, float("nan"), dtype=pos[0].dtype, device="cuda")
    pdn.pdn_slot_fwd(*pos, Sd, A=Ad, gate=gate, precond=precond, knorm=knorm, o=o, **opt, **KW, **kw)
    torch.cuda.synchronize()
    return host(o), host(Sd), host(Ad)


def want(b, S, A, lens, gate, precond, src=None, dst=None, fresh=None, knorm="none"):
    N = len(lens)
    src = range(N) if src is None else src
    dst = src if dst is None else dst
    starts = np.concatenate([[0], np.cumsum(lens)])
    o, S1, A1 = np.full(b["v"].shape, np.nan), S.copy(), None if A is None else A.copy()
    for n in range(N):
        if not (0 <= src[n] < len(S) and 0 <= dst[n] < len(S)):
            continue
        s, a = S[src[n]], None if A is None else A[src[n]]
        if fresh is not None and fresh[n]:
            s, a = 0 * s, None if a is None else 0 * a
        rows = np.arange(starts[n], starts[n + 1])
        o[rows], s, a = tokens(b, rows, s, a, gate, precond, knorm)
        S1[dst[n]] = s
        if A is not None:
            A1[dst[n]] = a
    return o, S1, A1, starts


def check(got, ref, io, T, what=""):
    """Values against the oracle's; what the call has to leave alone is left alone, NaN marks included."""
    (o, S, A), (ro, rS, rA) = got, ref
    bo, bs = bars(io, T)
    assert np.array_equal(np.isnan(o), np.isnan(ro)), what
    live = ~np.isnan(ro)
    e = [rel_err(o[live], ro[live]) if live.any() else 0.0, rel_err(S, rS), rel_err(A, rA) if A is not None else 0.0]
    print(what, "o %.2e S %.2e A %.2e" % tuple(e))
    assert e[0] <= bo and e[1] <= bs and e[2] <= bs, (what, e)


CASES = [
    # (io, gate, precond, knorm, H, Hk, dk, dv, lens)
    ("bf16", "scalar", "squash", "none", 2, 2, 128, 128, [1]),
    ("bf16", "scalar", "identity", "none", 4, 2, 128, 128, [1, 1, 1, 1, 1]),
    ("bf16", "channel", "squash", "none", 2, 1, 128, 128, [1, 1, 1]),
    ("f32", "none", "external", "none", 3, 3, 64, 64, [1, 1]),
    ("bf16", "channel", "diag_sm", "none", 2, 2, 64, 128, [1, 1]),
    ("f32", "channel", "atq", "none", 2, 2, 128, 64, [1, 1]),
    ("bf16", "scalar", "squash", "beta", 2, 2, 128, 128, [1, 1]),
    ("bf16", "scalar", "squash", "none", 2, 2, 128, 128, [2]),
    ("bf16", "scalar", "squash", "none", 3, 1, 128, 128, [8, 0, 5, 1, 4]),
    ("f32", "scalar", "identity", "none", 4, 2, 128, 128, [7, 3, 8]),
    ("f32", "channel", "squash", "none", 2, 2, 64, 64, [6, 8, 2]),
    ("bf16", "channel", "external", "none", 2, 1, 128, 64, [8, 3]),
    ("bf16", "none", "squash", "m", 2, 2, 64, 128, [5, 8]),
    ("bf16", "scalar", "squash", "beta", 2, 2, 128, 128, [3, 8]),
    ("bf16", "channel", "squash", "1pm", 2, 2, 128, 128, [7]),
    ("f32", "scalar", "diag_sm", "none", 2, 2, 128, 64, [8, 6]),
    ("bf16", "scalar", "atq", "none", 2, 2, 128, 128, [8, 4]),
    ("f32", "channel", "atq", "none", 2, 2, 64, 128, [5]),
    ("bf16", "scalar", "squash", "none", 2, 2, 128, 128, [9, 16, 17, 0, 1]),
    ("bf16", "scalar", "squash", "none", 4, 2, 128, 128, [130, 63, 64, 65, 31, 33]),
    ("bf16", "none", "identity", "none", 2, 1, 128, 128, [257, 100]),
    ("bf16", "channel", "squash", "none", 2, 2, 128, 128, [97, 40, 64]),
    ("f32", "scalar", "squash", "none", 2, 2, 64, 64, [129, 1, 32]),
    ("f32", "none", "external", "none", 2, 1, 128, 128, [70]),
    ("f32", "channel", "diag_sm", "none", 2, 2, 64, 128, [45, 90]),
    ("bf16", "scalar", "diag_sm", "none", 2, 2, 128, 64, [45, 90]),
    ("bf16", "none", "atq", "none", 2, 2, 128, 128, [66, 129]),
    ("bf16", "channel", "atq", "none", 2, 2, 128, 128, [66, 129]),
    ("bf16", "scalar", "squash", "m", 2, 2, 64, 128, [66]),
    ("bf16", "channel", "identity", "none", 6, 2, 64, 64, [100, 7, 200]),
    ("bf16", "scalar", "external", "none", 4, 2, 64, 128, [100, 7, 200]),
    # whole blocks of eight, and one token past them
    ("f32", "scalar", "squash", "none", 2, 2, 128, 128, [16, 24, 32, 40]),
    ("f32", "channel", "identity", "none", 2, 1, 128, 128, [17, 25, 8, 41]),
    ("f32", "none", "atq", "none", 2, 2, 128, 128, [24, 9]),
    ("f32", "channel", "atq", "none", 2, 2, 128, 128, [33, 16]),
    ("f32", "scalar", "squash", "beta", 2, 1, 64, 128, [32, 15]),
    ("f32", "channel", "diag_sm", "none", 2, 2, 128, 64, [48, 1, 0, 31]),
    ("bf16", "channel", "squash", "none", 4, 2, 128, 128, [16, 24, 32, 40]),
    # the split products' 32: whole chunks, one short, one past
    ("bf16", "scalar", "squash", "none", 2, 2, 128, 128, [32, 64, 96]),
    ("bf16", "scalar", "identity", "none", 2, 2, 64, 64, [95, 97, 31]),
]


@pytest.mark.parametrize("io,gate,precond,knorm,H,Hk,dk,dv,lens", CASES)
def test_rule(io, gate, precond, knorm, H, Hk, dk, dv, lens):
    """Ragged sequences in permuted slots; the other slots stay bit for bit."""
    rng = np.random.default_rng(len(lens) * 1000 + sum(lens))
    N, M = len(lens), sum(lens)
    b = batch(rng, M, H, Hk, dk, dv, io, gate, precond)
    S, A = pool(rng, N + 2, H, dk, dv, precond)
    src = rng.permutation(N + 2)[:N]
    o, S1, A1, starts = want(b, S, A, lens, gate, precond, src, knorm=knorm)
    got = run(b, S, A, io, gate, precond, strided=M % 2 == 1, knorm=knorm, starts=i32(starts), slots=i32(src),
              max_tokens=max(lens))
    check(got, (o, S1, A1), io, max(lens), f"{io}/{gate}/{precond}/{knorm} {lens}")
    rest = np.setdiff1d(np.arange(N + 2), src)
    assert np.array_equal(got[1][rest], S[rest])
    if A is not None:
        assert np.array_equal(got[2][rest], A[rest])


@pytest.mark.parametrize("io,gate,precond", [("bf16", "scalar", "identity"), ("bf16", "none", "external"),
                                              ("bf16", "channel", "identity"), ("f32", "scalar", "external")])
def test_heads_whole_and_in_halves(io, gate, precond):
    """129 heads are a workgroup each, 128 two of half the columns: the same values,
    in place, and with a fork and a new sequence among them."""
    rng = np.random.default_rng(129)
    N, H, d, lens = 43, 3, 128, [11 + n % 24 for n in range(43)]
    b = batch(rng, sum(lens), H, H, d, d, io, gate, precond)
    S, A = pool(rng, N + 1, H, d, d, precond)
    src, fresh = list(range(N)), [int(n == 5) for n in range(N)]
    dst = [N if n == 7 else n for n in range(N)]
    o, S1, A1, starts = want(b, S, A, lens, gate, precond, src, dst, fresh)
    whole = run(b, S, A, io, gate, precond, starts=i32(starts), slots=i32(src), slots_out=i32(dst), fresh=i32(fresh),
                max_tokens=max(lens))
    check(whole, (o, S1, A1), io, max(lens))
    n = 42   # 126 heads
    part = run(b, S, A, io, gate, precond, starts=i32(starts[:n + 1]), slots=i32(src[:n]), slots_out=i32(dst[:n]),
               fresh=i32(fresh[:n]), max_tokens=max(lens))
    o[starts[n]:] = np.nan
    S1[n - N - 1] = S[n - N - 1]
    check(part, (o, S1, A1), io, max(lens))


@pytest.mark.parametrize("T", [1, 6, 50])
def test_forks_fresh_padding(T):
    """Two sequences read one slot and write others; one is new; one has no
    slot, whose rows stay as they were; rows behind the last sequence too."""
    rng = np.random.default_rng(T)
    H, d, lens = 2, 128, [T, T, max(T - 1, 1), T]
    b = batch(rng, sum(lens) + 3, H, H, d, d, "bf16", "scalar", "squash")
    S, A = pool(rng, 8, H, d, d, "squash")
    src, dst, fresh = [5, 5, 1, -1], [0, 2, 1, 3], [0, 0, 1, 0]
    o, S1, A1, starts = want(b, S, A, lens, "scalar", "squash", src, dst, fresh)
    S_in, A_in = S.copy(), A.copy()
    S_in[1], A_in[1] = np.nan, np.inf   # a fresh sequence reads nothing of its slot
    got = run(b, S_in, A_in, "bf16", "scalar", "squash", starts=i32(starts), slots=i32(src), slots_out=i32(dst),
              fresh=i32(fresh), max_tokens=T)
    check(got, (o, S1, A1), "bf16", T)
    assert np.array_equal(got[1][[3, 4, 5, 6, 7]], S[[3, 4, 5, 6, 7]])
    # a slot past the pool, either way, is no slot
    for kw in (dict(slots=i32([0, 8, 2, 3])), dict(slots=i32([0, 1, 2, 3]), slots_out=i32([0, 2 ** 30, 2, 3]))):
        o, S1, A1, _ = want(b, S, A, lens, "scalar", "squash", [0, -1, 2, 3])
        check(run(b, S, A, "bf16", "scalar", "squash", starts=i32(starts), max_tokens=T, **kw), (o, S1, A1), "bf16", T)


@pytest.mark.parametrize("T", [1, 5, 40])
def test_even_rows_without_lists(T):
    """No starts, no slots: sequence n is rows n T .. of slot n."""
    rng = np.random.default_rng(40 + T)
    b = batch(rng, 3 * T, 2, 2, 64, 64, "f32", "none", "identity")
    S, A = pool(rng, 4, 2, 64, 64, "identity")
    o, S1, A1, _ = want(b, S, A, [T] * 3, "none", "identity")
    check(run(b, S, A, "f32", "none", "identity", max_tokens=T), (o, S1, A1), "f32", T)


@pytest.mark.parametrize("T", [1, 7, 90])
def test_rows_cut_and_clamped(T):
    """A sequence longer than max_tokens is cut; starts outside the tensors are
    clamped to them, and a range that runs backwards is empty."""
    rng = np.random.default_rng(60 + T)
    M = 3 * T + 2
    b = batch(rng, M, 2, 2, 64, 64, "bf16", "scalar", "identity")
    S, A = pool(rng, 4, 2, 64, 64, "identity")
    starts = [-7, T + 1, 2 ** 31 - 1, T, M + 50]
    ranges = [(0, T), (T + 1, 2 * T + 1), (0, 0), (T, 2 * T)]   # (the last overlaps the second: rows of equal value either way)
    starts[3] = 2 * T + 1
    ranges[3] = (2 * T + 1, min(3 * T + 1, M))
    o, S1 = np.full(b["v"].shape, np.nan), S.copy()
    for n, (lo, hi) in enumerate(ranges):
        o[lo:hi], S1[n], _ = tokens(b, np.arange(lo, hi), S[n], None, "scalar", "identity")
    got = run(b, S, A, "bf16", "scalar", "identity", starts=i32(starts), max_tokens=T)
    check(got, (o, S1, None), "bf16", T)


def test_pieces_equal_the_whole():
    """A prompt and then single tokens and pieces: the states carry over, as
    one run over all tokens would."""
    rng = np.random.default_rng(5)
    H, d, total = 2, 128, 120
    for gate in ("scalar", "channel"):
        b = batch(rng, total, H, H, d, d, "bf16", gate, "squash")
        S, A = pool(rng, 1, H, d, d, "squash")
        o, S1, A1, _ = want(b, S, A, [total], gate, "squash")
        at, outs, s, a = 0, [], S, A
        for n in (70, 1, 1, 8, 3, 37):
            part = {k: None if x is None else x[at:at + n] for k, x in b.items()}
            r = run(part, s, a, "bf16", gate, "squash", max_tokens=n)
            outs.append(r[0])
            s, a, at = r[1], r[2], at + n
        check((np.concatenate(outs), s, a), (o, S1, A1), "bf16", total, gate)


@pytest.mark.parametrize("T", [1, 8, 60])
def test_strong_decay_and_zero_keys(T):
    """Log-decays of -9 a token, zero keys, zero write strengths; and decays to
    zero without the per-channel gate, where nothing bounds them."""
    rng = np.random.default_rng(80 + T)
    for gate, strength in (("channel", 7.0), ("scalar", 400.0)):
        b = batch(rng, 2 * T, 2, 2, 128, 128, "f32", gate, "squash", strength=0.0)
        b["g"] = np.clip(-strength * rng.random(b["g"].shape), -9.0 if gate == "channel" else -400.0, 0.0)
        b["g"] = b["g"].astype(np.float32).astype(np.float64)
        b["k"][::3] = 0.0
        b["beta"][1::4] = 0.0
        S, A = pool(rng, 2, 2, 128, 128, "squash")
        A[1] = 0.0
        o, S1, A1, starts = want(b, S, A, [T, T], gate, "squash")
        check(run(b, S, A, "f32", gate, "squash", starts=i32(starts), max_tokens=T), (o, S1, A1), "f32", T, gate)


@pytest.mark.parametrize("T", [1, 8, 60])
@pytest.mark.parametrize("io", ["bf16", "f32"])
def test_state_forgotten(T, io):
    """Log-decays of -inf, of the lowest value and of -1e5 (a document's first
    token): nothing comes through, and the tokens after keep their small decays."""
    rng = np.random.default_rng(85 + T)
    low = [-np.inf, float(np.finfo(np.float32).min), -1e5]
    b = batch(rng, 3 * T, 2, 2, 128, 128, io, "scalar", "squash")
    for n in range(3):
        for t in {0, T // 3, T // 2, T - 1}:
            b["g"][n * T + t, n % 2] = low[(n + t) % 3]
            b["g_p"][n * T + t, 1] = low[n]
    S, A = pool(rng, 3, 2, 128, 128, "squash")
    o, S1, A1, starts = want(b, S, A, [T] * 3, "scalar", "squash")
    assert np.isfinite(S1).all()
    check(run(b, S, A, io, "scalar", "squash", starts=i32(starts), max_tokens=T), (o, S1, A1), io, T)


@pytest.mark.parametrize("T", [1, 6, 70])
def test_two_streams_at_once(T):
    """Calls on two streams, each with its own half of a pool, their outputs and
    workspaces allocated by the calls; and the same pool's halves in one call."""
    import torch
    import paper_2604_21100_amd as pdn
    rng = np.random.default_rng(95 + T)
    N, H, d = 4, 4, 128
    b = batch(rng, N * T, H, H, d, d, "bf16", "scalar", "squash")
    S, A = pool(rng, N, H, d, d, "squash")
    ref = want(b, S, A, [T] * N, "scalar", "squash")
    pos, opt = dev_batch(b, "bf16", "squash")
    Sd, Ad = dev(S), dev(A)
    cut = lambda x, lo: x if x is None or x.dim() == 1 else x[lo * T:(lo + 2) * T]   # noqa: E731
    lists = [i32([0, 1]), i32([2, 3])]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    outs = [pdn.pdn_slot_fwd(*[cut(x, 2 * i) for x in pos], Sd, A=Ad, gate="scalar", slots=lists[i], max_tokens=T,
                             starts=None, stream=streams[i], **{n: cut(x, 2 * i) for n, x in opt.items()}, **KW)
            for i in range(2)]
    torch.cuda.synchronize()
    check((np.concatenate([host(x) for x in outs]), host(Sd), host(Ad)), ref[:3], "bf16", T)
    check(run(b, S, A, "bf16", "scalar", "squash", max_tokens=T), ref[:3], "bf16", T)


@pytest.mark.parametrize("T", [1, 8, 100])
def test_nan_stays_in_its_sequence(T):
    """A sequence with NaN values does not reach its neighbours or other slots."""
    rng = np.random.default_rng(90 + T)
    b = batch(rng, 3 * T, 2, 2, 128, 128, "bf16", "scalar", "squash")
    S, A = pool(rng, 3, 2, 128, 128, "squash")
    o, S1, A1, starts = want(b, S, A, [T] * 3, "scalar", "squash")
    b["v"][T:2 * T] = np.nan
    b["k"][T:2 * T] = np.inf
    go, gS, gA = run(b, S, A, "bf16", "scalar", "squash", starts=i32(starts), max_tokens=T)
    keep = np.r_[0:T, 2 * T:3 * T]
    check((go[keep], gS[[0, 2]], gA[[0, 2]]), (o[keep], S1[[0, 2]], A1[[0, 2]]), "bf16", T)
    assert np.isnan(go[T:2 * T]).all() and np.isnan(gS[1]).any()


@pytest.mark.parametrize("T", [1, 8, 100])
def test_graph_and_streams(T):
    """A captured call replayed on new contents, with eager work of its own
    between; and a call on a side stream."""
    import torch
    import paper_2604_21100_amd as pdn
    rng = np.random.default_rng(100 + T)
    H, d, N = 4, 128, 3
    sets = []
    for _ in range(3):
        b = batch(rng, N * T, H, 2, d, d, "bf16", "scalar", "squash")
        S, A = pool(rng, N, H, d, d, "squash")
        lens = [T, max(T // 2, 1), T - 1]
        sets.append((b, S, A, lens, want(b, S, A, lens, "scalar", "squash")))
    b, S, A, lens, _ = sets[0]
    pos, opt = dev_batch(b, "bf16", "squash")
    Sd, Ad, o, starts = dev(S), dev(A), torch.empty_like(pos[2]), i32([0] * (N + 1))
    call = lambda: pdn.pdn_slot_fwd(*pos, Sd, A=Ad, gate="scalar", starts=starts, max_tokens=T, o=o, **opt, **KW)   # noqa: E731
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for b, S, A, lens, (ro, rS, rA, rs) in sets + sets[:1]:
        p2, o2 = dev_batch(b, "bf16", "squash")
        for x, y in zip(pos, p2):
            x.copy_(y)
        for n, x in opt.items():
            if x is not None:
                x.copy_(o2[n])
        Sd.copy_(dev(S))
        Ad.copy_(dev(A))
        starts.copy_(i32(rs))
        o.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        check((host(o), host(Sd), host(Ad)), (ro, rS, rA), "bf16", T)


def test_more_than_2_31_elements():
    """Slots and rows whose offsets pass 32 bits."""
    import torch
    import paper_2604_21100_amd as pdn
    rng = np.random.default_rng(7)
    H, d = 16, 128
    P = 2 ** 31 // (H * d * d) + 9   # the last slots start past 2^31 elements (8.6 GB)
    M, gap = 66, 2 ** 25   # rows 2^25 elements apart: the last starts past 2^31
    b = batch(rng, M, H, H, d, d, "bf16", "none", "identity")
    S, _ = pool(rng, 2, H, d, d, "identity")
    o, S1, _, _ = want(b, S, None, [M - 1, 1], "none", "identity")
    big = torch.zeros(P, H, d, d, device="cuda")
    big[P - 1], big[3] = dev(S[0]), dev(S[1])
    pos, opt = dev_batch(b, "bf16", "identity")
    wide = torch.empty((M - 1) * gap + H * d, dtype=torch.bfloat16, device="cuda").as_strided((M, H, d), (gap, d, 1))
    wide.copy_(pos[2])
    kw = dict(gate="none", precond="identity", starts=i32([0, M - 1, M]), slots=i32([P - 1, 3]), max_tokens=M)
    got = pdn.pdn_slot_fwd(pos[0], pos[1], wide, pos[3], big, **kw, **KW)
    torch.cuda.synchronize()
    check((host(got), host(big[[P - 1, 3]]), None), (o, S1, None), "bf16", M)


def test_refusals_of_the_binding():
    import torch
    import paper_2604_21100_amd as pdn
    rng = np.random.default_rng(1)
    b = batch(rng, 4, 2, 2, 64, 64, "bf16", "none", "identity")
    (q, k, v, beta), _ = dev_batch(b, "bf16", "identity")
    S = torch.zeros(4, 2, 64, 64, device="cuda")
    kw = dict(precond="identity")
    pdn.pdn_slot_fwd(q, k, v, beta, S, **kw)
    for bad, err in ((dict(beta=beta[:3]), ValueError), (dict(beta=beta.double()), TypeError),
                     (dict(k=k.float()), TypeError), (dict(v=v[..., :32]), ValueError),
                     (dict(v=v.transpose(0, 1).contiguous().transpose(0, 1)), ValueError),
                     (dict(S=S.transpose(2, 3)), ValueError), (dict(S=S.cpu()), ValueError),
                     (dict(slots=torch.zeros(4, dtype=torch.int64, device="cuda")), TypeError),
                     (dict(starts=torch.zeros(3, dtype=torch.int32, device="cuda"), slots=i32([0] * 4)), ValueError),
                     (dict(S=S[:3].contiguous()), pdn.PdnError),           # four sequences, three slots
                     (dict(A=torch.zeros(4, 2, 64, device="cuda")), pdn.PdnError)):
        a = dict(dict(q=q, k=k, v=v, beta=beta, S=S), **bad)
        with pytest.raises(err):
            pdn.pdn_slot_fwd(a.pop("q"), a.pop("k"), a.pop("v"), a.pop("beta"), a.pop("S"), **kw, **a)
    torch.cuda.synchronize()

