"""The state-pool calls on the host: what they refuse, before any HIP call
(fake addresses, never dereferenced; every call here fails validation or has
nothing to do)."""
import ctypes

import pytest

pdn = pytest.importorskip("paper_2604_21100_amd", reason="libpdn.so not built")

A = 1 << 28   # fake addresses this far apart do not overlap


def prob(**kw):
    return pdn.make_problem(**dict(dict(B=3, T=8, H=4, dk=128, dv=64, gate="scalar", precond="squash"), **kw))


def inputs(**kw):
    v = dict(q=A, k=2 * A, v=3 * A, beta=4 * A, g=5 * A, beta_p=6 * A, g_p=7 * A, log_a_scale=8 * A, A0=None, S0=None,
             ktilde=None)
    v.update(kw)
    return pdn.Inputs(*[v[n] for n, _ in pdn.Inputs._fields_])


def slots(draft=True, **kw):
    v = dict(tokens=20, slots=5, Hk=2, q_stride=0, k_stride=0, v_stride=0, starts=9 * A, slot=10 * A, slot_out=11 * A,
             fresh=12 * A, S=13 * A, A=14 * A, tape=15 * A if draft else None, tape_tokens=8 if draft else 0,
             pending=16 * A if draft else None, accepted=17 * A if draft else None)
    v.update(kw)
    return pdn.Slots(*[v[n] for n, _ in pdn.Slots._fields_])


def call(draft, p=None, i=None, s=None, o=18 * A):
    fn = pdn._lib.pdn_slot_draft if draft else pdn._lib.pdn_slot_fwd
    p, i, s = p or prob(), i or inputs(), s or slots(draft)
    return fn(ctypes.byref(p), ctypes.byref(i), ctypes.byref(s), o, None)


@pytest.mark.parametrize("draft", [False, True])
def test_refusals(draft):
    S = lambda **kw: slots(draft, **kw)   # noqa: E731
    cases = [
        (dict(p=prob(dk=96)), pdn.PDN_ERR_UNSUPPORTED), (dict(p=prob(B=-1)), pdn.PDN_ERR_SHAPE),
        (dict(p=prob(x=0.5)), pdn.PDN_ERR_VALUE), (dict(p=prob(precond="diag_sm", ridge=0.0)), pdn.PDN_ERR_VALUE),
        (dict(s=S(tokens=-1)), pdn.PDN_ERR_SHAPE), (dict(s=S(slots=-1)), pdn.PDN_ERR_SHAPE),
        (dict(s=S(Hk=3)), pdn.PDN_ERR_SHAPE), (dict(s=S(Hk=8)), pdn.PDN_ERR_SHAPE), (dict(s=S(Hk=-2)), pdn.PDN_ERR_SHAPE),
        (dict(s=S(tokens=1 << 31)), pdn.PDN_ERR_SHAPE), (dict(s=S(slots=1 << 31)), pdn.PDN_ERR_SHAPE),
        (dict(p=prob(B=1 << 23)), pdn.PDN_ERR_SHAPE), (dict(p=prob(B=1 << 20)), pdn.PDN_ERR_SHAPE),   # B H of 2^22
        (dict(s=S(starts=None)), pdn.PDN_ERR_SHAPE),                  # 3 x 8 rows are not 20
        (dict(s=S(slot=None, slots=2)), pdn.PDN_ERR_SHAPE),           # three sequences, two slots
        (dict(s=S(q_stride=255)), pdn.PDN_ERR_SHAPE), (dict(s=S(q_stride=260)), pdn.PDN_ERR_ALIGN),
        (dict(s=S(k_stride=257)), pdn.PDN_ERR_ALIGN), (dict(s=S(v_stride=128)), pdn.PDN_ERR_SHAPE),
        (dict(s=S(q_stride=1 << 62)), pdn.PDN_ERR_SHAPE),
        (dict(s=S(k_stride=(1 << 25) + 8)), pdn.PDN_ERR_SHAPE), (dict(p=prob(H=1 << 22), s=S(Hk=0)), pdn.PDN_ERR_SHAPE),
        (dict(i=inputs(q=None)), pdn.PDN_ERR_NULL), (dict(i=inputs(beta=None)), pdn.PDN_ERR_NULL), (dict(o=None), pdn.PDN_ERR_NULL),
        (dict(i=inputs(g=None)), pdn.PDN_ERR_NULL), (dict(i=inputs(beta_p=None)), pdn.PDN_ERR_NULL),
        (dict(i=inputs(log_a_scale=None)), pdn.PDN_ERR_NULL), (dict(s=S(S=None)), pdn.PDN_ERR_NULL),
        (dict(s=S(A=None)), pdn.PDN_ERR_NULL), (dict(p=prob(precond="external"), s=S(A=None)), pdn.PDN_ERR_NULL),
        (dict(p=prob(gate="none")), pdn.PDN_ERR_VALUE), (dict(i=inputs(S0=30 * A)), pdn.PDN_ERR_VALUE),
        (dict(i=inputs(A0=30 * A)), pdn.PDN_ERR_VALUE), (dict(p=prob(precond="identity")), pdn.PDN_ERR_VALUE),
        (dict(i=inputs(q=A + 8)), pdn.PDN_ERR_ALIGN), (dict(s=S(S=13 * A + 4)), pdn.PDN_ERR_ALIGN),
        (dict(s=S(starts=9 * A + 2)), pdn.PDN_ERR_ALIGN), (dict(o=18 * A + 2), pdn.PDN_ERR_ALIGN),
        (dict(o=A), pdn.PDN_ERR_ALIAS), (dict(o=13 * A), pdn.PDN_ERR_ALIAS), (dict(s=S(A=13 * A + 64)), pdn.PDN_ERR_ALIAS),
        (dict(s=S(slot=13 * A)), pdn.PDN_ERR_ALIAS),
        (dict(i=inputs(q=18 * A - 4096), s=S(q_stride=4096)), pdn.PDN_ERR_ALIAS),   # a strided row reaches o
    ]
    if draft:
        cases += [(dict(s=S(tape_tokens=7)), pdn.PDN_ERR_SHAPE), (dict(s=S(tape_tokens=1 << 40)), pdn.PDN_ERR_SHAPE),
                  (dict(s=S(tape_tokens=0), p=prob(T=0)), pdn.PDN_ERR_SHAPE), (dict(s=S(tape=None)), pdn.PDN_ERR_NULL),
                  (dict(s=S(pending=None)), pdn.PDN_ERR_NULL), (dict(s=S(tape=13 * A)), pdn.PDN_ERR_ALIAS),
                  (dict(s=S(accepted=16 * A)), pdn.PDN_ERR_ALIAS), (dict(s=S(pending=16 * A + 4)), pdn.PDN_ERR_ALIGN)]
    else:
        cases += [(dict(s=S(tape=15 * A)), pdn.PDN_ERR_VALUE), (dict(s=S(pending=16 * A)), pdn.PDN_ERR_VALUE),
                  (dict(s=S(accepted=17 * A)), pdn.PDN_ERR_VALUE)]
    for kw, status in cases:
        assert call(draft, **kw) == status, (kw, status)
    fn = pdn._lib.pdn_slot_draft if draft else pdn._lib.pdn_slot_fwd
    p, i, s = prob(), inputs(), S()
    assert fn(None, ctypes.byref(i), ctypes.byref(s), 18 * A, None) == pdn.PDN_ERR_NULL
    assert fn(ctypes.byref(p), None, ctypes.byref(s), 18 * A, None) == pdn.PDN_ERR_NULL
    assert fn(ctypes.byref(p), ctypes.byref(i), None, 18 * A, None) == pdn.PDN_ERR_NULL


@pytest.mark.parametrize("draft", [False, True])
def test_nothing_to_do(draft):
    """No sequences, heads or slots: success without a launch (no GPU here)."""
    assert call(draft, p=prob(B=0)) == pdn.PDN_OK
    assert call(draft, s=slots(draft, slots=0)) == pdn.PDN_OK
    assert call(draft, p=prob(H=0), s=slots(draft, Hk=0)) == pdn.PDN_OK


def verify(N=3, rows=9, V=50, dtype=pdn.PDN_F32, p=A, q=2 * A, ids=3 * A, u=4 * A, r=5 * A, starts=6 * A,
           accepted=7 * A, token=8 * A, ws=9 * A, ws_bytes=None):
    if ws_bytes is None:
        ws_bytes = 1 << 20
    return pdn._lib.pdn_draft_verify(N, rows, V, dtype, p, q, ids, u, r, starts, accepted, token, ws, ws_bytes, None)


def test_verify_refusals():
    for kw, status in [
            (dict(N=-1), pdn.PDN_ERR_SHAPE), (dict(rows=-1), pdn.PDN_ERR_SHAPE), (dict(V=-1), pdn.PDN_ERR_SHAPE),
            (dict(V=0), pdn.PDN_ERR_SHAPE), (dict(rows=10, starts=None), pdn.PDN_ERR_SHAPE),
            (dict(N=1 << 24), pdn.PDN_ERR_SHAPE), (dict(N=1 << 24, V=0, rows=0), pdn.PDN_ERR_SHAPE), (dict(V=1 << 31), pdn.PDN_ERR_SHAPE), (dict(rows=1 << 31), pdn.PDN_ERR_SHAPE),
            (dict(dtype=7), pdn.PDN_ERR_DTYPE), (dict(p=None), pdn.PDN_ERR_NULL), (dict(ids=None), pdn.PDN_ERR_NULL),
            (dict(u=None), pdn.PDN_ERR_NULL), (dict(r=None), pdn.PDN_ERR_NULL), (dict(accepted=None), pdn.PDN_ERR_NULL),
            (dict(token=None), pdn.PDN_ERR_NULL), (dict(p=A + 2), pdn.PDN_ERR_ALIGN),
            (dict(dtype=pdn.PDN_BF16, q=2 * A + 1), pdn.PDN_ERR_ALIGN), (dict(ids=3 * A + 2), pdn.PDN_ERR_ALIGN),
            (dict(token=7 * A + 8), pdn.PDN_ERR_ALIAS), (dict(accepted=3 * A), pdn.PDN_ERR_ALIAS),
            (dict(ws=A), pdn.PDN_ERR_ALIAS), (dict(ws=None), pdn.PDN_ERR_WORKSPACE),
            (dict(ws_bytes=8), pdn.PDN_ERR_WORKSPACE), (dict(ws=9 * A + 128), pdn.PDN_ERR_WORKSPACE)]:
        assert verify(**kw) == status, (kw, status)
    assert verify(N=0) == pdn.PDN_OK
    with pytest.raises(pdn.PdnError):
        pdn.pdn_draft_verify_workspace_size(-1, 5)
    assert pdn._lib.pdn_draft_verify_workspace_size(1, 5, None) == pdn.PDN_ERR_NULL
    assert pdn.pdn_draft_verify_workspace_size(2, 131072) >= 2 * 64 * 16


def test_record_size():
    assert pdn.pdn_tape_record(128, 64, "scalar", "identity") == 128 + 64 + 4
    assert pdn.pdn_tape_record(128, 64, "channel", "squash") == 3 * 128 + 64


def test_host_tensors_are_refused():
    """The compiled part of the binding, without a GPU: what it says of tensors on the
    host, of wrong kinds and dimensions."""
    torch = pytest.importorskip("torch")
    z = torch.zeros
    rows, S = z(4, 2, 64), z(4, 2, 64, 64)
    good = dict(q=rows, k=rows, v=rows, beta=z(4, 2), S=S)
    for bad, err in ((dict(), ValueError), (dict(S=S[0]), ValueError), (dict(q=rows[0]), ValueError),
                     (dict(q=None), TypeError), (dict(v=[1.0]), TypeError)):
        a = dict(good, **bad)
        with pytest.raises(err):
            pdn.pdn_slot_fwd(a["q"], a["k"], a["v"], a["beta"], a["S"], precond="identity")
        with pytest.raises(err):
            pdn.pdn_slot_draft(a["q"], a["k"], a["v"], a["beta"], a["S"], z(4, 1, 2, 132), z(4, 2, dtype=torch.int32),
                               precond="identity")
    with pytest.raises(KeyError):
        pdn.pdn_slot_fwd(rows, rows, rows, z(4, 2), S, precond="none of them")
    i = z(4, dtype=torch.int32)
    for p, err in ((z(4, 9), ValueError), (z(4), ValueError), (None, (TypeError, AttributeError))):
        with pytest.raises(err):
            pdn.pdn_draft_verify(p, i, z(4), z(2))
