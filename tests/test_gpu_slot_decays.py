"""Per-channel log-decays of any size: a channel that forgets between two tokens of a block, or
in all of them, beside channels that keep everything; with write keys of any size.

Bars are those of the state-pool tests: a decay over up to seven tokens is a product of as many
exponentials, each within 2^-22, which the bars' 1e-5 holds many times over."""
import numpy as np
import pytest

from slot_util import KW, batch, dev, dev_batch, host, i32, pool, tokens
from test_gpu_slots import bars, check, rel_err, run, want

pytestmark = pytest.mark.gpu

LOW = [0.0, -1e-4, -0.1, -3.0, -12.0, -30.0, -86.0, -90.0, -200.0, -1e5, float(np.finfo(np.float32).min), -np.inf]


@pytest.mark.parametrize("io,precond,dk,dv", [("f32", "squash", 128, 128), ("bf16", "identity", 128, 64),
                                              ("bf16", "external", 64, 128), ("f32", "diag_sm", 64, 64),
                                              ("bf16", "atq", 128, 128)])
@pytest.mark.parametrize("T", [1, 2, 3, 5, 8, 9, 60])
def test_any_decay(io, precond, dk, dv, T):
    """Every kind of log-decay in every place."""
    rng = np.random.default_rng(T * 100 + dk + dv)
    lens = [T, max(T - 1, 1), T]
    b = batch(rng, sum(lens), 2, 2, dk, dv, io, "channel", precond)
    b["g"] = np.asarray(LOW, np.float32).astype(np.float64)[rng.integers(0, len(LOW), b["g"].shape)]
    b["g"][:, 1] = np.where(rng.random(b["g"][:, 1].shape) < 0.8, -0.05, b["g"][:, 1])   # a head that mostly keeps
    S, A = pool(rng, 3, 2, dk, dv, precond)
    o, S1, A1, starts = want(b, S, A, lens, "channel", precond)
    assert np.isfinite(S1).all()
    check(run(b, S, A, io, "channel", precond, starts=i32(starts), max_tokens=T), (o, S1, A1), io, T, f"{precond} {T}")


@pytest.mark.parametrize("T", [2, 8, 9, 40])
@pytest.mark.parametrize("total", [-60.0, -84.5, -500.0])
def test_large_write_keys(T, total):
    """A channel's log-decays of eight tokens that add up to `total`, write keys in the hundreds."""
    rng = np.random.default_rng(T)
    b = batch(rng, 2 * T, 2, 2, 128, 128, "f32", "channel", "external")
    b["g"][:] = np.float32(total / 8)
    b["g"][:, :, ::3] = -0.01
    b["ktilde"] *= 4096.0
    b["beta"] = (2.0 ** -12 * b["beta"]).astype(np.float32).astype(np.float64)
    S, A = pool(rng, 2, 2, 128, 128, "external")
    o, S1, A1, starts = want(b, S, A, [T, T], "channel", "external")
    check(run(b, S, A, "f32", "channel", "external", starts=i32(starts), max_tokens=T), (o, S1, A1), "f32", T)


@pytest.mark.parametrize("precond", ["squash", "identity", "atq"])
@pytest.mark.parametrize("T", [2, 8, 20])
def test_any_decay_of_drafts(T, precond):
    """Outputs of drafted tokens, and the state with some of them accepted.  A record has the
    sum of its log-decays (each counting as -128 at the least) in fp32, so the state's bar
    grows with that sum: a decay is the exponential of a difference of two, 2^-23 of them,
    and at most T updates count."""
    import torch
    import paper_2604_21100_amd as pdn
    rng = np.random.default_rng(7 * T)
    P, H, d = 3, 2, 128
    b = batch(rng, P * T, H, H, d, d, "f32", "channel", precond)
    b["g"] = np.asarray(LOW, np.float32).astype(np.float64)[rng.integers(0, len(LOW), b["g"].shape)]
    S, A = pool(rng, P, H, d, d, precond)
    Sd, Ad = dev(S), dev(A)
    tape = torch.full((P, T, H, pdn.pdn_tape_record(d, d, "channel", precond)), float("nan"), device="cuda")
    pending = torch.zeros(P, H, dtype=torch.int32, device="cuda")
    pos, opt = dev_batch(b, "f32", precond)
    kw = dict(A=Ad, gate="channel", precond=precond, max_tokens=T, **opt, **KW)
    o = host(pdn.pdn_slot_draft(*pos, Sd, tape, pending, starts=i32([n * T for n in range(P + 1)]), **kw))
    acc = [T, T - 1, 1]
    pdn.pdn_slot_draft(*pos, Sd, tape, pending, accepted=i32(acc), starts=i32([0] * (P + 1)), **kw)
    bo, _ = bars("f32", T)
    for n in range(P):
        rows = np.arange(n * T, (n + 1) * T)
        ro = tokens(b, rows, S[n], None if A is None else A[n], "channel", precond)[0]
        _, s, a = tokens(b, rows[:acc[n]], S[n], None if A is None else A[n], "channel", precond)
        G = np.abs(np.maximum(b["g"][rows[:acc[n]]], -128.0).sum(0)).max()
        e = rel_err(o[rows], ro), rel_err(host(Sd)[n], s)
        print(precond, T, n, e, G)
        assert e[0] <= bo and e[1] <= 1e-5 + T * 2.0 ** -23 * G


@pytest.mark.parametrize("T", [3, 8, 21])
@pytest.mark.parametrize("gate", ["scalar", "channel"])
def test_a_record_rounds_its_sum_once(gate, T):
    """The summed log-decay of a pending token is within half a step, 2^-24 of it, of the
    exact sum (a little more where that itself is taken in 64 bits)."""
    import torch
    import paper_2604_21100_amd as pdn
    rng = np.random.default_rng(T)
    P, H, d = 2, 2, 128
    b = batch(rng, P * T, H, H, d, d, "f32", gate, "identity", strength=1.0)
    b["g"][::4] = (30.0 * b["g"][::4]).astype(np.float32).astype(np.float64)
    b["g"] = np.maximum(b["g"], -128.0)
    tape = torch.full((P, T, H, pdn.pdn_tape_record(d, d, gate, "identity")), float("nan"), device="cuda")
    pos, opt = dev_batch(b, "f32", "identity")
    pdn.pdn_slot_draft(*pos, torch.zeros(P, H, d, d, device="cuda"), tape, torch.zeros(P, H, dtype=torch.int32, device="cuda"),
                       gate=gate, precond="identity", max_tokens=T, **opt, **KW)
    G = np.cumsum(b["g"].reshape(P, T, H, -1), 1)
    off = np.abs(host(tape)[..., 2 * d:2 * d + (d if gate == "channel" else 4)] - G) / np.abs(G)
    print(gate, T, "%.3f half steps" % (off.max() * 2 ** 24))
    assert off.max() <= 2.0 ** -24 * (1 + 2.0 ** -20)
