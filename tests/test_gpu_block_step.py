"""The calls around the rule together with it, as a block has them: a training step's gradients
against the same chain in 64 bits, and decoding token by token against the prompt's call."""
import numpy as np
import pytest

import block_util as bu
from gpu_util import rel_err

pytestmark = pytest.mark.gpu
EPS = 1e-6


def test_training_step():
    """x -> norm -> projection -> unit q, k -> rule -> gated norm -> projection -> residual and norm, and back, in fp32
    against 64 bits (the oracle's recurrence and adjoint in the middle).  Bars: the rule's own of its fp32 tests, 1e-4."""
    import torch
    import paper_2604_21100_amd as pdn
    from oracle import abi
    rng = np.random.default_rng(1)
    B, T, H, d = 2, 70, 2, 64
    D = H * d
    f = lambda *s: rng.standard_normal(s).astype(np.float32).astype(np.float64)   # noqa: E731
    x, wn, wo, w2, scale = f(B, T, D), 1 + 0.2 * f(D), 1 + 0.2 * f(d), 1 + 0.2 * f(D), 0.5 + 0.1 * f(D)
    Wi, Wo = f(D, 4 * D) / 8, f(D, D) / 8
    wn, wo, w2, scale, Wi, Wo = (a.astype(np.float32).astype(np.float64) for a in (wn, wo, w2, scale, Wi, Wo))
    beta, g = 1 / (1 + np.exp(-f(B, T, H))), -0.1 * np.logaddexp(0, f(B, T, H))
    beta_p, g_p, las = 1 / (1 + np.exp(-f(B, T, H))), -0.1 * np.logaddexp(0, f(B, T, H)), 0.3 * f(H)
    beta, g, beta_p, g_p, las = (a.astype(np.float32).astype(np.float64) for a in (beta, g, beta_p, g_p, las))
    du2, dh2 = f(B, T, D), f(B, T, D)
    e = float(np.float32(EPS))

    # in 64 bits
    flat = lambda a: a.reshape(-1, D)   # noqa: E731
    (u, _), (h, _) = bu.rnorm(flat(x), None, wn, False, None, None, 1.0, e)
    proj = (u @ Wi).reshape(B, T, 4, H, d)
    q0, k0, v, z = (proj[:, :, i] for i in range(4))
    q, k = (bu.hnorm(a, "l2", None, None, "none", e)[0] for a in (q0, k0))
    inp = dict(q=q, k=k, v=v, beta=beta, g=g, beta_p=beta_p, g_p=g_p, log_a_scale=las, A0=None, S0=None)
    o = np.moveaxis(abi.forward(inp, gate="scalar", B=B, H=H)["o"].reshape(B, H, T, d), 1, 2)
    n = bu.hnorm(o, "rms", wo, z, "silu", e)[0]
    y = n.reshape(-1, D) @ Wo
    (u2, _), (h2, _) = bu.rnorm(y, flat(x), w2, True, None, scale, 0.5, e)
    r = {m: a[0] for m, a in bu.rnorm_bwd(flat(du2), flat(dh2), h2, y, w2, True, None, scale, 0.5, e).items()}
    dn = (r["dy"] @ Wo.T).reshape(B, T, H, d)
    s = {m: a[0] for m, a in bu.hnorm_bwd(dn, o, "rms", wo, z, "silu", e).items()}
    inp["dO"] = s["dx"]
    c = abi.backward(inp, gate="scalar", B=B, H=H)
    at = lambda a: np.moveaxis(np.asarray(a).reshape(B, H, T, -1), 1, 2)   # noqa: E731
    dq, dk = (bu.hnorm_bwd(at(c[m]), a, "l2", None, None, "none", e)["dx"][0] for m, a in (("dq", q0), ("dk", k0)))
    dproj = np.stack([dq, dk, at(c["dv"]), s["dz"]], 2).reshape(-1, 4 * D)
    t = {m: a[0] for m, a in bu.rnorm_bwd(dproj @ Wi.T, r["dresidual"], flat(x), None, wn, False, None, None, 1.0, e).items()}
    want = dict(u2=u2, h2=h2, dx=t["dresidual"], dwn=t["dweight"], dwo=s["dweight"], dw2=r["dweight"], dscale=r["dscale"],
                dWi=u.T @ dproj, dWo=n.reshape(-1, D).T @ r["dy"], dbeta=at(c["dbeta"])[..., 0], dg=at(c["dg"])[..., 0])

    # the framework's calls
    dev = lambda a: torch.tensor(a, dtype=torch.float32, device="cuda")   # noqa: E731
    X, Wi_, Wo_ = dev(x), dev(Wi), dev(Wo)
    vec = {m: dev(a) for m, a in dict(wn=wn, wo=wo, w2=w2, scale=scale).items()}
    U, _ = pdn.pdn_residual_norm(X, weight=vec["wn"], eps=EPS, want_h=False)
    P = (U.view(-1, D) @ Wi_).view(B, T, 4 * D)
    Q0, K0, V, Z = (a.unflatten(-1, (H, d)) for a in P.split(D, -1))
    Q, K = pdn.pdn_head_norm(Q0, norm="l2", eps=EPS), pdn.pdn_head_norm(K0, norm="l2", eps=EPS)
    kw = dict(g=dev(g), gate="scalar", beta_p=dev(beta_p), g_p=dev(g_p), log_a_scale=dev(las))
    prob = pdn.make_problem(B, T, H, d, d, io="f32", gate="scalar")
    ws = torch.empty(pdn.pdn_workspace_size(prob, True), dtype=torch.uint8, device="cuda")
    Vc, Be = V.contiguous(), dev(beta)
    O = pdn.pdn_chunk_fwd(Q, K, Vc, Be, workspace=ws, train=True, **kw)[0]
    N = pdn.pdn_head_norm(O, weight=vec["wo"], z=Z, eps=EPS)
    Y = (N.view(-1, D) @ Wo_).view(B, T, D)
    late = dict(weight=vec["w2"], post_norm=True, scale=vec["scale"], alpha=0.5, eps=EPS)
    U2, H2 = pdn.pdn_residual_norm(Y, X, **late)
    R = pdn.pdn_residual_norm_bwd(dev(du2), H2, Y, dh=dev(dh2), **late)
    DN = (R["dy"].view(-1, D) @ Wo_.T).view(B, T, H, d)
    DP = torch.empty_like(P)
    DQ0, DK0, DV, DZ = (a.unflatten(-1, (H, d)) for a in DP.split(D, -1))
    S = pdn.pdn_head_norm_bwd(DN, O, weight=vec["wo"], z=Z, eps=EPS, outputs=dict(dz=DZ))
    C = pdn.pdn_chunk_bwd(Q, K, Vc, Be, S["dx"], workspace=ws, saved=True, **kw)
    DV.copy_(C["dv"])
    pdn.pdn_head_norm_bwd(C["dq"], Q0, norm="l2", eps=EPS, outputs=dict(dx=DQ0))
    pdn.pdn_head_norm_bwd(C["dk"], K0, norm="l2", eps=EPS, outputs=dict(dx=DK0))
    DU = (DP.view(-1, 4 * D) @ Wi_.T).view(B, T, D)
    L = pdn.pdn_residual_norm_bwd(DU, X, dh=R["dresidual"], weight=vec["wn"], eps=EPS)
    got = dict(u2=U2, h2=H2, dx=L["dresidual"], dwn=L["dweight"], dwo=S["dweight"], dw2=R["dweight"], dscale=R["dscale"],
               dWi=U.view(-1, D).T @ DP.view(-1, 4 * D), dWo=N.view(-1, D).T @ R["dy"].view(-1, D), dbeta=C["dbeta"], dg=C["dg"])
    for m, a in want.items():
        err = rel_err(got[m].double().cpu().numpy().reshape(a.shape), a)
        print(m, "%.1e" % err)
        assert err <= 1e-4, (m, err)


def test_decoding_token_by_token():
    """The block over a prompt in one call and token by token from a pool: the rows' calls give the same bits for the same
    rows however many there are, and the rule its own bars."""
    import torch
    import paper_2604_21100_amd as pdn
    torch.manual_seed(2)
    T, H, d = 9, 4, 64
    D = H * d
    r = lambda *s: torch.randn(s, device="cuda")   # noqa: E731
    x, w, Wi, Wo = r(T, D), 1 + 0.1 * r(D), r(D, 4 * D) / 16, r(D, D) / 16
    beta, g = torch.sigmoid(r(T, H)), -0.1 * torch.nn.functional.softplus(r(T, H))

    def block(rows, S, n):
        u, _ = pdn.pdn_residual_norm(x[rows], weight=w, want_h=False)
        proj = u @ Wi
        q, k, v, z = (a.unflatten(-1, (H, d)) for a in proj.split(D, -1))
        pdn.pdn_head_norm(q, norm="l2", y=q)   # in the projection's rows
        pdn.pdn_head_norm(k, norm="l2", y=k)
        o = pdn.pdn_slot_fwd(q, k, v, beta[rows].contiguous(), S, starts=torch.tensor([0, n], dtype=torch.int32, device="cuda"),
                             max_tokens=n, g=g[rows].contiguous(), gate="scalar", precond="identity")
        y = pdn.pdn_head_norm(o, weight=w[:d].contiguous(), z=z, y=o).view(-1, D) @ Wo
        h = x[rows].clone()
        return pdn.pdn_residual_norm(y, h, weight=w, alpha=0.5, h=h)

    S1 = torch.zeros(1, H, d, d, device="cuda")
    u1, h1 = block(slice(0, T), S1, T)
    S2, outs = torch.zeros_like(S1), []
    for t in range(T):
        outs.append(block(slice(t, t + 1), S2, 1))
    for i, whole in enumerate((u1, h1)):
        got = torch.cat([o[i] for o in outs])
        assert rel_err(got.double().cpu().numpy(), whole.double().cpu().numpy()) <= 1e-4
    assert rel_err(S2.double().cpu().numpy(), S1.double().cpu().numpy()) <= 1e-4
    a, _ = pdn.pdn_residual_norm(x, weight=w)
    assert torch.equal(a[4:5], pdn.pdn_residual_norm(x[4:5], weight=w)[0])


def test_speculating_rounds_in_a_graph():
    """A layer of a speculating server from the residual stream to the next token and the counts, captured once: rounds of
    replays give the bits of eager rounds on copies of the same states, other eager calls between them."""
    import torch
    import paper_2604_21100_amd as pdn
    torch.manual_seed(3)
    N, K, H, d, V, P = 3, 4, 2, 64, 3001, 4
    M, D, dev = N * K, H * d, "cuda"
    r = lambda *s: torch.randn(s, device=dev)   # noqa: E731
    i32 = lambda *a: torch.tensor(a, dtype=torch.int32, device=dev)   # noqa: E731
    embed, Wi, Wo, head = r(V, D), r(D, 4 * D) / 11, r(D, D) / 11, r(D, V) / 4
    w, wo, temperature, rep = 1 + 0.1 * r(D), 1 + 0.1 * r(d), torch.tensor([0.0, 0.7, 1.2], device=dev), torch.full((N,), 1.2, device=dev)
    starts, slots = i32(0, K, 2 * K, 3 * K), i32(2, 0, 3)

    class Server:
        def __init__(self):
            self.S, self.tape = torch.zeros(P, H, d, d, device=dev), torch.zeros(P, K, H, pdn.pdn_tape_record(d, d, "scalar", "identity"), device=dev)
            self.pending, self.counts = torch.zeros(P, H, dtype=torch.int32, device=dev), torch.zeros(P, V, dtype=torch.int32, device=dev)
            self.accepted, self.token = torch.zeros(N, dtype=torch.int32, device=dev), torch.zeros(N, dtype=torch.int32, device=dev)
            self.ids, self.beta, self.g = torch.zeros(M, dtype=torch.int32, device=dev), torch.rand(M, H, device=dev), -torch.rand(M, H, device=dev)
            self.u, self.r, self.p = torch.rand(M, device=dev), torch.rand(N, device=dev), torch.zeros(M, V, device=dev)

        def step(self):
            h = embed[self.ids.long()]
            u, _ = pdn.pdn_residual_norm(h, weight=w, want_h=False)
            q, k, v, z = (a.unflatten(-1, (H, d)) for a in (u @ Wi).split(D, -1))
            pdn.pdn_head_norm(q, norm="l2", y=q)
            pdn.pdn_head_norm(k, norm="l2", y=k)
            o = pdn.pdn_slot_draft(q, k, v, self.beta, self.S, self.tape, self.pending, accepted=self.accepted, starts=starts, slots=slots,
                                   max_tokens=K, g=self.g, gate="scalar", precond="identity")
            y = pdn.pdn_head_norm(o, weight=wo, z=z, y=o).view(M, D) @ Wo
            u, _ = pdn.pdn_residual_norm(y, h, weight=w, alpha=0.5, h=h)
            pdn.pdn_logits(u @ head, temperature=temperature, repetition=rep, counts=self.counts, slots=slots, ids=self.ids, starts=starts, out=self.p)
            pdn.pdn_draft_verify(self.p, self.ids, self.u, self.r, starts=starts, accepted=self.accepted, token=self.token)
            pdn.pdn_token_counts(self.ids, self.counts, starts=starts, slots=slots, accepted=self.accepted)

    a, b = Server(), Server()
    for m in ("beta", "g"):
        getattr(b, m).copy_(getattr(a, m))
    warm = Server()
    warm.step()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        b.step()
    for turn in range(5):
        ids = torch.randint(0, 40, (M,), dtype=torch.int32, device=dev)
        ids[::K] = a.token.clamp(min=0)
        u, t = torch.rand(M, device=dev) * 0.1, torch.rand(N, device=dev)
        for s in (a, b):
            s.ids.copy_(ids)
            s.u.copy_(u)
            s.r.copy_(t)
        a.step()
        g.replay()
        warm.step()
        torch.cuda.synchronize()
        for m in ("S", "tape", "pending", "counts", "accepted", "token", "p"):
            assert torch.equal(getattr(a, m), getattr(b, m)), (turn, m)
    assert a.counts.sum() >= 5 * N and (a.p.sum(1) - 1).abs().max() < 1e-5
