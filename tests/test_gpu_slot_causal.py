"""NaN and infinities in a token: the outputs of the tokens before it, of other heads, and
of what it does not touch are those of a batch without it.

Bars are those of the state-pool tests."""
import numpy as np
import pytest

from slot_util import KW, batch, dev, dev_batch, host, i32, pool, tokens
from test_gpu_slots import bars, rel_err, run

pytestmark = pytest.mark.gpu

FORMS = [("bf16", "scalar", "squash", 128, 8), ("f32", "channel", "external", 64, 6), ("bf16", "channel", "atq", 128, 7),
         ("f32", "scalar", "squash", 64, 40), ("bf16", "channel", "identity", 128, 37), ("bf16", "scalar", "diag_sm", 128, 30),
         ("bf16", "scalar", "squash", 128, 70), ("bf16", "scalar", "identity", 64, 64), ("bf16", "none", "external", 128, 45)]
DRAFTS = [("bf16", "scalar", "squash", 128, 8), ("bf16", "channel", "identity", 128, 5), ("f32", "scalar", "atq", 64, 12)]


def places(T):
    """First, last, and around the sixteens and thirty-twos of a chunk."""
    return sorted({0, 1, T // 2, T - 1} | {t for t in (4, 7, 8, 15, 16, 23, 31, 32, 63) if t < T})


def spoil(b, kind, t, value):
    x = b[kind]
    if kind == "v":
        x[t, 0, 5] = value          # one column
    elif x.ndim == 3:
        x[t, 0, 3] = value          # one channel
    else:
        x[t, 0] = value


@pytest.mark.parametrize("draft,io,gate,precond,d,T",
                         [(False, *f) for f in FORMS] + [(True, *f) for f in DRAFTS])
def test_only_what_comes_after(draft, io, gate, precond, d, T):
    import torch
    import paper_2604_21100_amd as pdn
    rng = np.random.default_rng(T + d)
    H = 2
    clean = batch(rng, T, H, H, d, d, io, gate, precond)
    S, A = pool(rng, 1, H, d, d, precond)
    ro, rS, _ = tokens(clean, np.arange(T), S[0], None if A is None else A[0], gate, precond)
    bo, bs = bars(io, T)
    kinds = [k for k in ("v", "k", "q", "beta", "g", "ktilde", "beta_p", "g_p") if clean[k] is not None]
    for kind in kinds:
        for value in (np.nan, np.inf):
            if value == np.inf and kind in ("g", "g_p"):
                continue
            for t in places(T):
                b = {n: None if x is None else x.copy() for n, x in clean.items()}
                spoil(b, kind, t, value)
                if draft:
                    pos, opt = dev_batch(b, io, precond)
                    Sd, Ad = dev(S), dev(A)
                    tape = torch.full((1, T, H, pdn.pdn_tape_record(d, d, gate, precond)), float("nan"), device="cuda")
                    o = host(pdn.pdn_slot_draft(*pos, Sd, tape, torch.zeros(1, H, dtype=torch.int32, device="cuda"), A=Ad,
                                                gate=gate, precond=precond, max_tokens=T, **opt, **KW))
                    assert np.array_equal(host(Sd), S)
                else:
                    o, gS, _ = run(b, S, A, io, gate, precond, starts=i32([0, T]), max_tokens=T)
                    assert rel_err(gS[0, 1], rS[1]) <= bs
                live = np.ones(o.shape, bool)
                if kind == "q":
                    live[t, 0] = False
                elif kind == "v":
                    live[t:, 0, 5] = False
                else:
                    live[t:, 0] = False
                what = (kind, value, t)
                assert np.isfinite(o[live]).all(), what
                assert rel_err(o[live], ro[live]) <= bo, what
                if kind not in ("beta_p", "g_p"):
                    assert not np.isfinite(o[t, 0, 5]), what
                if kind in ("v", "k", "beta", "g") and not (precond == "atq" and kind == "k"):
                    assert not np.isfinite(o[t:, 0, 5]).any(), what
