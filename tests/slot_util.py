"""Helpers of the state-pool tests: a random pool and packed batch, and what
the calls have to do to it in 64 bits (the oracle's token recurrence, sequence
by sequence)."""
import numpy as np

import pdn_inputs as pi
from oracle import recurrent

GRAM = ("squash", "diag_sm", "atq")
KW = dict(x=1.5, scale=0.7, ridge=0.5)


def unit(z):
    return z / np.linalg.norm(z, axis=-1, keepdims=True)


def batch(rng, M, H, Hk, dk, dv, io, gate, precond, strength=0.1):
    """M packed tokens, as float64 arrays of what the device sees."""
    rnd = pi.round_bf16 if io == "bf16" else (lambda z: z.astype(np.float32))
    f32 = lambda z: z.astype(np.float32).astype(np.float64)   # noqa: E731
    decay = lambda *s: f32(-strength * np.logaddexp(0, rng.standard_normal(s)))   # noqa: E731
    b = dict(q=rnd(unit(rng.standard_normal((M, Hk, dk)))), k=rnd(unit(rng.standard_normal((M, Hk, dk)))),
             v=rnd(rng.standard_normal((M, H, dv))), beta=f32(2.0 / (1 + np.exp(-rng.standard_normal((M, H))))),
             g=None, beta_p=None, g_p=None, ktilde=None)
    if gate != "none":
        b["g"] = decay(M, H) if gate == "scalar" else decay(M, H, dk)
    if precond in GRAM:
        b["beta_p"], b["g_p"] = f32(1 / (1 + np.exp(-rng.standard_normal((M, H))))), decay(M, H)
    if precond == "external":
        b["ktilde"] = rnd(b["k"] * rng.uniform(1 / 1.5, 1.5, b["k"].shape))
    return {n: None if x is None else x.astype(np.float64) for n, x in b.items()}


def pool(rng, P, H, dk, dv, precond):
    S = (0.3 * rng.standard_normal((P, H, dk, dv))).astype(np.float32).astype(np.float64)
    A = np.exp(rng.standard_normal((P, H, dk)) - 3.0).astype(np.float32).astype(np.float64) if precond in GRAM else None
    return S, A


def las(H):
    return (0.3 * np.sin(1.0 + np.arange(H))).astype(np.float32).astype(np.float64)


def tokens(b, rows, S, A, gate, precond, knorm="none"):
    """The recurrence over `rows` of the batch from S [H, dk, dv], A [H, dk]: o [n, H, dv], S, A."""
    H, Hk = b["v"].shape[1], b["q"].shape[1]
    if len(rows) == 0:
        return np.zeros((0, H, b["v"].shape[2])), S, A
    head = lambda x: None if x is None else np.moveaxis(x[rows], 1, 0)   # noqa: E731
    rep = lambda x: None if x is None else head(np.repeat(x, H // Hk, axis=1))   # noqa: E731
    r = recurrent.pdn_forward(
        rep(b["q"]), rep(b["k"]), head(b["v"]), head(b["beta"]), g=head(b["g"]), gate=gate, precond=precond,
        beta_p=head(b["beta_p"]), g_p=head(b["g_p"]), mu=np.exp(las(H)), kt_ext=rep(b["ktilde"]),
        S0=np.swapaxes(S, 1, 2), A0=A, knorm=knorm, **KW)
    return np.moveaxis(r["o"], 0, 1), np.swapaxes(r["S_T"], 1, 2), r["A_T"]


def dev(x, dtype=None, strided=False):
    """To the device; strided: as a slice of wider rows."""
    import torch
    if x is None:
        return None
    t = torch.from_numpy(np.ascontiguousarray(x)).to(dtype or torch.float32).cuda()
    if not strided or not t.numel():
        return t
    wide = torch.full((t.shape[0], t[0].numel() + 64), float("nan"), dtype=t.dtype, device="cuda")
    flat = wide[:, 32:32 + t.shape[1] * t.shape[2]]
    flat.copy_(t.reshape(t.shape[0], -1))
    return flat.unflatten(1, t.shape[1:])


def dev_batch(b, io, precond, strided=False):
    """q, k, v, beta and the keyword tensors of a call."""
    import torch
    dt = torch.bfloat16 if io == "bf16" else torch.float32
    pos = [dev(b[n], dt, strided) for n in "qkv"] + [dev(b["beta"])]
    kw = dict(g=dev(b["g"]), beta_p=dev(b["beta_p"]), g_p=dev(b["g_p"]), ktilde=dev(b["ktilde"], dt),
              log_a_scale=dev(las(b["v"].shape[1])) if precond == "squash" else None)
    return pos, kw


def i32(x):
    import torch
    return None if x is None else torch.tensor(list(x), dtype=torch.int32, device="cuda")


def host(t):
    return None if t is None else t.float().cpu().numpy().astype(np.float64)
