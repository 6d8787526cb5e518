"""What pdn_slot_fwd and pdn_slot_draft put into o, where its terms cancel: o is then
as exact as its fp32 terms are, and only its own rounding is to io.

Bars.  Every case leaves two terms of o that are not zero, x and y, of about the same size
m, and o = x - y is a small part of it.  With fp32 operands and sums, a term is off by
what its factors are, and the sum by some roundings of 2^-24 m; eight are allowed, 2^-21 m.
Factors: a state element and a correction beta v are exact to one rounding; a decay
e^g, |g| < 1, is off by a rounding of its argument and one unit of the exponential, 2^-22;
a write key's gain by 2^-21 (logarithm, reciprocal and exponential of one unit each,
all of slope below one).  Outputs are rounded to io once: bf16 2^-8 of the value."""
import numpy as np
import pytest

from slot_util import KW, dev, dev_batch, host, i32, pool, tokens

pytestmark = pytest.mark.gpu

H, D = 2, 128


def plain_batch(T, v, beta, g=None):
    """T tokens with the keys e_0, e_1, .., which do not see each other's."""
    f = lambda x: np.asarray(x, np.float32).astype(np.float64)   # noqa: E731
    k = np.zeros((T, H, D))
    k[np.arange(T), :, np.arange(T)] = 1.0
    return dict(q=np.zeros((T, H, D)), k=k, v=v, beta=f(beta), g=None if g is None else f(g), beta_p=None, g_p=None,
                ktilde=None)


def pairs(rng, T, among):
    """q rows e_a - e_b, with a and b of the first among(t) channels."""
    q = np.zeros((T, H, D))
    for t in range(T):
        for h in range(H):
            if among(t) > 1:
                a, b = rng.permutation(among(t))[:2]
                q[t, h, a], q[t, h, b] = 1.0, -1.0
    return q


def check(b, S, A, io, gate, precond, T, size, off, draft=False):
    """|o - exact| <= a rounding to io + off * size, value by value."""
    import torch
    import paper_2604_21100_amd as pdn
    pos, opt = dev_batch(b, io, precond)
    Sd, Ad = dev(S), dev(A)
    kw = dict(A=Ad, gate=gate, precond=precond, starts=i32([0, T]), max_tokens=T, **opt, **KW)
    if draft:
        tape = torch.full((1, T, H, pdn.pdn_tape_record(D, D, gate, precond)), float("nan"), device="cuda")
        o = pdn.pdn_slot_draft(*pos, Sd, tape, torch.zeros(1, H, dtype=torch.int32, device="cuda"), **kw)
    else:
        o = pdn.pdn_slot_fwd(*pos, Sd, **kw)
    ref = tokens(b, np.arange(T), S[0], None if A is None else A[0], gate, precond)[0]
    excess = np.abs(host(o) - ref) - (2.0 ** -8 if io == "bf16" else 0.0) * np.abs(ref)
    print(io, gate, precond, T, "largest |o| %.2e, off %.2e (bar %.2e)" % (np.abs(ref).max(), excess.max(), off * size))
    assert np.abs(ref).max() < 2.0 ** -6 * size and np.abs(ref).max() > 4 * off * size
    assert excess.max() <= off * size


FORMS = [("bf16", "identity", 16), ("bf16", "squash", 40), ("bf16", "external", 16), ("bf16", "identity", 6),
         ("f32", "identity", 16), ("bf16", "identity", 1)]


@pytest.mark.parametrize("io,precond,T", FORMS)
@pytest.mark.parametrize("gate", ["none", "channel"])
def test_the_state_under_the_queries(io, precond, T, gate):
    """Rows of the state that differ in their last twelve bits; no writes, no decay."""
    rng = np.random.default_rng(T)
    S, A = pool(rng, 1, H, D, D, precond)
    base = 1.0 + rng.random((1, H, 1, D))
    S = (base + 2.0 ** -12 * rng.random((1, H, D, D))).astype(np.float32).astype(np.float64)
    b = plain_batch(T, np.zeros((T, H, D)), np.zeros((T, H)), np.zeros((T, H, D)) if gate == "channel" else None)
    b["q"] = pairs(rng, T, lambda t: D)
    if precond == "external":
        b["ktilde"] = b["k"].copy()
    if precond == "squash":
        b["beta_p"], b["g_p"] = np.zeros((T, H)), np.zeros((T, H))
    check(b, S, A, io, gate, precond, T, 2.0, 2.0 ** -21)


@pytest.mark.parametrize("io,precond,T", FORMS[:5])
@pytest.mark.parametrize("draft", [False, True])
def test_corrections(io, precond, T, draft):
    """Corrections e_s = beta_s v that differ in their last bits."""
    rng = np.random.default_rng(20 + T)
    S, A = pool(rng, 1, H, D, D, precond)
    v = np.broadcast_to(np.round(64 * (1 + rng.random((1, 1, D)))) / 64, (T, H, D))   # (bf16 numbers)
    b = plain_batch(T, v, 0.75 + 2.0 ** -10 * rng.random((T, H)))
    b["q"] = pairs(rng, T, lambda t: t + 1)
    if precond == "external":
        b["ktilde"] = b["k"].copy()
    off = 2.0 ** -21
    if precond == "squash":   # (every channel with the same preconditioner state, so the same gain)
        A[:] = 1.0
        b["beta_p"], b["g_p"] = np.zeros((T, H)), np.zeros((T, H))
        off = 2.0 ** -20
    check(b, 0 * S, A, io, "none", precond, T, 2.0, off, draft)


@pytest.mark.parametrize("io,precond,T", [("bf16", "identity", 16), ("bf16", "identity", 30), ("bf16", "identity", 7),
                                          ("f32", "identity", 16)])
@pytest.mark.parametrize("gate", ["scalar", "channel"])
def test_decays(io, precond, T, gate):
    """Decays that differ in their last bits, over equal corrections."""
    rng = np.random.default_rng(40 + T)
    S, _ = pool(rng, 1, H, D, D, precond)
    v = np.broadcast_to(np.round(64 * (1 + rng.random((1, 1, D)))) / 64, (T, H, D))
    g = -2.0 ** -12 * rng.random((T, H))
    b = plain_batch(T, v, np.ones((T, H)), g if gate == "scalar" else np.repeat(g[:, :, None], D, 2))
    b["q"] = pairs(rng, T, lambda t: t + 1)
    # (an exponential for the decay, where a channel's is a product of up to seven)
    check(b, 0 * S, None, io, gate, precond, T, 2.0, 2.0 ** -21 + (2 if gate == "scalar" else 7) * 2.0 ** -22)


@pytest.mark.parametrize("io,T", [("bf16", 16), ("bf16", 40), ("bf16", 8), ("f32", 16)])
def test_write_keys(io, T):
    """Write keys whose gains differ in their last bits: one key of ones, then none."""
    rng = np.random.default_rng(60 + T)
    S, A = pool(rng, 1, H, D, D, "squash")
    A = (1.0 + 2.0 ** -9 * rng.random(A.shape)).astype(np.float32).astype(np.float64)
    v = np.broadcast_to(np.round(64 * (1 + rng.random((1, 1, D)))) / 64, (T, H, D))
    b = plain_batch(T, v, np.ones((T, H)))
    b["k"][:] = 0.0
    b["k"][0] = 1.0
    b["q"] = pairs(rng, T, lambda t: D)
    b["beta_p"], b["g_p"] = np.zeros((T, H)), np.zeros((T, H))
    check(b, 0 * S, A, io, "none", "squash", T, 3.0, 2.0 ** -21 + 2 * 2.0 ** -21)
