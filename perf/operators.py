"""Serving from a pool of recurrent states: the calls, their plain forms and
what they have to return.

Three operators:

  slot_fwd   the gated delta rule over packed ragged sequences whose states
             live in slots of a pool: one token a sequence (decoding) or whole
             prompts
  draft      the same rule over a few drafted tokens: the tokens the last
             round accepted are applied to the state, the new ones are scored
             without moving it and left pending on the tape
  verify     the drafted tokens against the target's probabilities, from
             given random numbers: how many hold, and the token after them

Every state is read from one slot and written to another, so a pass can be
repeated.  Queries, keys and values are slices of one projection's rows,
as a layer has them; lengths are ragged, in random slots.

Tensors follow the layers' own setup: unit-norm queries and keys whose
channels differ in scale, sigmoid write strengths, log-decays -0.1 softplus,
values that are an association of the keys plus noise.
"""
import math
import random

import torch

own = False

_F32, _F64 = torch.float32, torch.float64
_X = 1.5
_C = 32          # tokens a chunk of the plain form


def _rule(kind, N, T, H, Hk, dk=128, dv=128, *, io="bf16", gate="scalar", precond="squash", name=None):
    c = dict(kind=kind, N=N, T=T, H=H, Hk=Hk, dk=dk, dv=dv, io=io, gate=gate, precond=precond)
    return c if name is None else dict(c, name=name)


def _verify(N, K, V, *, io="f32", q=True, name=None):
    c = dict(kind="verify", N=N, K=K, V=V, io=io, q=q)
    return c if name is None else dict(c, name=name)


def listed():
    return [
        # one user, one new token: the latency of a call
        _rule("decode", 1, 1, 16, 16, name="decode_n1_h16"),
        # a decoding server's ordinary step through the 1B-scale layer
        _rule("decode", 64, 1, 16, 16, name="decode_n64_h16"),
        # a full server: many sequences, two value heads to a key head, no preconditioner
        _rule("decode", 256, 1, 32, 16, precond="identity", name="decode_n256_h32_g2"),
        # a few short fp32 prompts through small heads: a user's test run
        _rule("prefill", 3, 333, 4, 4, 64, 64, io="f32", gate="none", name="prefill_f32_n3_t333_h4_d64"),
        # a batch of ragged prompts through the 1B-scale layer
        _rule("prefill", 16, 1000, 16, 16, name="prefill_n16_t1000_h16"),
        # longer prompts, shared key heads, no preconditioner
        _rule("prefill", 8, 2048, 32, 16, precond="identity", name="prefill_n8_t2048_h32_g2"),
        # prompts through the per-channel-gate layer
        _rule("prefill", 12, 700, 16, 16, gate="channel", name="prefill_channel_n12_t700_h16"),
        # one user with a few drafted tokens
        _rule("draft", 1, 5, 16, 16, name="draft_n1_t5_h16"),
        # a server verifying up to seven drafted tokens a sequence
        _rule("draft", 64, 8, 16, 16, name="draft_n64_t8_h16"),
        # the per-channel gate, shared key heads
        _rule("draft", 96, 4, 16, 8, gate="channel", precond="identity", name="draft_channel_n96_t4_h16_g2"),
        # one user's drafts against a mid-sized vocabulary, odd
        _verify(1, 4, 50257, name="verify_n1_k4_v50257"),
        # a server's drafts against a large vocabulary
        _verify(64, 7, 131072, name="verify_n64_k7_v131072"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of these ranges."""
    kind = rng.choice(("decode", "prefill", "prefill", "draft", "draft", "verify"))
    if kind == "verify":
        N, K = _log_int(rng, 1, 64), rng.randint(1, 7)
        return _verify(N, K, _log_int(rng, 1000, 131072), io=rng.choice(("f32", "f32", "bf16")), q=rng.random() < 0.7)
    H = rng.choice((1, 2, 4, 6, 8, 12, 16, 16, 32))
    Hk = H // rng.choice([d for d in (1, 1, 1, 2, 3, 4) if H % d == 0])
    dk, dv = rng.choice(((128, 128), (128, 128), (128, 128), (64, 64), (64, 128), (128, 64)))
    opt = dict(io="f32" if rng.random() < 0.2 else "bf16", gate=rng.choice(("none", "scalar", "scalar", "channel")),
               precond=rng.choice(("squash", "identity")))
    if kind == "decode":
        return _rule(kind, _log_int(rng, 1, 8192 // H), 1, H, Hk, dk, dv, **opt)
    if kind == "draft":
        return _rule(kind, _log_int(rng, 1, 1024 // H), rng.randint(2, 8), H, Hk, dk, dv, **opt)
    N = _log_int(rng, 1, 16)
    return _rule(kind, N, _log_int(rng, 2, min(2048, 262_144 // (N * H))), H, Hk, dk, dv, **opt)


def _lengths(c):
    """The sequences' rows, by the case alone (prepare() shuffles them): one of the most a sequence has, the others up
    to that; drafts are two rows or more, prompts may be empty, and a verification is of none to K drafts."""
    if c["kind"] == "verify":
        most, least = c["K"] + 1, 1
    else:
        most, least = c["T"], {"decode": 1, "draft": 2, "prefill": 0}[c["kind"]]
    rng = random.Random(c["N"] * 100_003 + most)
    return [most] + [rng.randint(least, most) for _ in range(c["N"] - 1)]


def _starts(c, gen):
    lens = torch.tensor(_lengths(c), device="cuda")[torch.randperm(c["N"], generator=gen, device="cuda")]
    s = torch.zeros(c["N"] + 1, dtype=torch.int64, device="cuda")
    s[1:] = torch.cumsum(lens, 0)
    return s


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed) * 7919 + 29)
    c = case
    if c["kind"] == "verify":
        return _prepare_verify(c, gen)
    N, T, H, Hk, dk, dv = (c[n] for n in ("N", "T", "H", "Hk", "dk", "dv"))
    io = torch.bfloat16 if c["io"] == "bf16" else _F32

    def normal(*shape):
        return torch.randn(shape, generator=gen, device="cuda", dtype=_F32)

    def ints(lo, hi, *shape):
        return torch.randint(lo, hi, shape, generator=gen, device="cuda")

    def unit(z):
        return z / z.norm(dim=-1, keepdim=True)

    def decay(*shape):
        return -0.1 * torch.nn.functional.softplus(normal(*shape))

    starts, M = _starts(c, gen), sum(_lengths(c))
    scale = torch.exp(0.5 * normal(1, Hk, dk))
    qk = [unit(normal(M, Hk, dk) * scale) for _ in range(2)]
    W = normal(H, dk, dv)
    kh = qk[1].to(io).float().repeat_interleave(H // Hk, 1)
    v = 0.8 * torch.matmul(kh.transpose(0, 1), W).transpose(0, 1) + 0.6 * normal(M, H, dv)
    # the three are slices of one projection's rows
    rows = torch.cat([t.reshape(M, -1).to(io) for t in (*qk, v)], 1)
    q, k, v = rows.split([Hk * dk, Hk * dk, H * dv], 1)
    d = dict(case=c, T=T, starts=starts.to(torch.int32), q=q.view(M, Hk, dk), k=k.view(M, Hk, dk), v=v.view(M, H, dv),
             beta=torch.sigmoid(normal(M, H)), g=None, beta_p=None, g_p=None, log_a_scale=None, A=None, fresh=None)
    if c["gate"] != "none":
        d["g"] = decay(M, H) if c["gate"] == "scalar" else decay(M, H, dk)
    slots = torch.randperm(2 * N, generator=gen, device="cuda").to(torch.int32)
    d["slots"], d["slots_out"] = slots[:N].contiguous(), slots[N:].contiguous()
    d["S"] = 0.1 * normal(2 * N, H, dk, dv) + 0.3 * W
    squash = c["precond"] == "squash"
    if squash:
        d["beta_p"], d["g_p"] = torch.sigmoid(normal(M, H)), decay(M, H)
        d["log_a_scale"] = 0.3 * normal(H)
        d["A"] = torch.exp(0.5 * normal(2 * N, H, dk) - 3.0)
    if c["kind"] == "prefill":   # some prompts are new, some continue
        d["fresh"] = ints(0, 2, N).to(torch.int32)
    if c["kind"] == "draft":
        # the last round's tokens, pending: write key, correction, prefix of the log-decay, preconditioner state
        P, n_g = 2 * N, dk if c["gate"] == "channel" else 4
        G = torch.zeros(P, T, H, n_g, device="cuda")
        if c["gate"] == "scalar":
            G += torch.cumsum(decay(P, T, H, 1), 1)
        if c["gate"] == "channel":
            G = torch.cumsum(decay(P, T, H, dk), 1)
        rec = [unit(normal(P, T, H, dk)), 0.5 * normal(P, T, H, dv), G]
        if squash:
            rec.append(torch.exp(0.5 * normal(P, T, H, dk) - 3.0))
        d["tape"] = torch.cat(rec, -1)
        d["pending"] = ints(1, T + 1, P)[:, None].expand(P, H).to(torch.int32).contiguous()
        d["accepted"] = torch.minimum(ints(1, T + 1, N), d["pending"][d["slots"].long(), 0].long()).to(torch.int32)
    return d


def _prepare_verify(c, gen):
    N, V = c["N"], c["V"]
    starts, M = _starts(c, gen), sum(_lengths(c))
    io = _F32 if c["io"] == "f32" else torch.bfloat16
    logits = 2.5 * torch.randn(M, V, generator=gen, device="cuda")
    p = torch.softmax(logits, 1)
    # row t's draft was drawn from a smaller model's view of row t - 1
    near = torch.softmax(torch.roll(logits, 1, 0) + 0.4 * torch.randn(M, V, generator=gen, device="cuda"), 1)
    ids = torch.multinomial(near, 1, generator=gen)[:, 0]
    if not c["q"]:   # drafts without probabilities: the smaller model's likeliest token
        ids = near.argmax(1)
    del logits
    rand = torch.rand(M + N, generator=gen, device="cuda")
    return dict(case=c, starts=starts.to(torch.int32), p=p.to(io), q=near.to(io) if c["q"] else None, ids=ids.to(torch.int32),
                u=rand[:M].contiguous(), r=rand[M:].contiguous())


def run(d):
    kind = d["case"]["kind"]
    if own:
        return _own(d, kind)
    if kind == "verify":
        return _plain_verify(d)
    return _plain_rule(d)


def _own(d, kind):
    import paper_2604_21100_amd as pdn
    if kind == "verify":
        accepted, token = pdn.pdn_draft_verify(d["p"], d["ids"], d["u"], d["r"], q=d["q"], starts=d["starts"])
        return {"accepted": accepted, "token": token}
    c = d["case"]
    kw = dict(starts=d["starts"], slots=d["slots"], slots_out=d["slots_out"], max_tokens=d["T"], g=d["g"], gate=c["gate"],
              precond=c["precond"], beta_p=d["beta_p"], g_p=d["g_p"], log_a_scale=d["log_a_scale"], A=d["A"], x=_X)
    if kind != "draft":
        o = pdn.pdn_slot_fwd(d["q"], d["k"], d["v"], d["beta"], d["S"], fresh=d["fresh"], **kw)
        return _outputs(d, o)
    o = pdn.pdn_slot_draft(d["q"], d["k"], d["v"], d["beta"], d["S"], d["tape"], d["pending"], accepted=d["accepted"], **kw)
    return _outputs(d, o)


def _outputs(d, o):
    """The outputs: the tokens', and the state's pools."""
    out = {"o": o, "S": d["S"], "A": d["A"]}
    if d["case"]["kind"] == "draft":
        out.update(tape=d["tape"], pending=d["pending"])
    return {n: t for n, t in out.items() if t is not None}


# ---------------------------------------------------------------- plain forms
def _padded(d, C):
    """The tokens of the sequences, [N, T, ...] with T a whole number of
    chunks, the rows behind a sequence's end zero."""
    starts = d["starts"].long()
    T = -(-d["T"] // C) * C
    t = torch.arange(T, device=starts.device)
    live = t[None, :] < (starts[1:] - starts[:-1])[:, None]
    at = torch.where(live, starts[:-1, None] + t[None, :], 0)

    def take(x, heads=1):
        if x is None:
            return None
        y = x.float()[at] * live.view(*live.shape, *[1] * (x.dim() - 1))
        return y.repeat_interleave(heads, 2) if heads > 1 else y

    return take, at, live


def _write_keys(k, beta_p, g_p, log_a_scale, A):
    """k [N, H, C, dk], beta_p, g_p [N, H, C], A [N, H, dk]: the write keys and A after every token."""
    Gp = torch.cumsum(g_p, -1)
    D = torch.exp((Gp[..., :, None] - Gp[..., None, :]).clamp(max=0.0)).tril()
    At = torch.exp(Gp)[..., None] * A[:, :, None] + torch.matmul(D, beta_p[..., None] * k * k)
    r = torch.log(At.clamp(min=1e-37)) - torch.exp(log_a_scale)[None, :, None, None]
    return torch.exp(-math.log(_X) * r / (1.0 + r.abs())) * k, At


def _solve(L):
    """(I + L)^{-1} of strictly lower L, row after row."""
    C = L.shape[-1]
    M = torch.eye(C, device=L.device).expand(L.shape).clone()
    for t in range(1, C):
        M[..., t, :t] = -torch.matmul(L[..., t:t + 1, :t], M[..., :t, :t])[..., 0, :]
    return M


def _plain_chunk(q, k, kt, v, beta, G, S):
    """One chunk, [N, H, C, ...] from the states S [N, H, dk, dv] ([dk, dv] being S^T);
    G: inclusive prefix of the log-decay, [N, H, C, 1 or dk].  Returns o, the corrections E and the next S."""
    if G.shape[-1] == 1:
        D = torch.exp((G - G.transpose(-1, -2)).clamp(max=0.0))
        kk, qk = torch.matmul(k, kt.transpose(-1, -2)) * D, torch.matmul(q, kt.transpose(-1, -2)) * D
    else:
        back = (kt * torch.exp(-G)).transpose(-1, -2)
        kk, qk = torch.matmul(k * torch.exp(G), back), torch.matmul(q * torch.exp(G), back)
    lam = torch.exp(G)
    X = beta[..., None] * (v - torch.matmul(k * lam, S))
    E = torch.matmul(_solve(torch.tril(beta[..., None] * kk, -1)), X)
    o = torch.matmul(q * lam, S) + torch.matmul(torch.tril(qk), E)
    end = G[..., -1:, :]
    S = torch.exp(end).transpose(-1, -2) * S + torch.matmul((kt * torch.exp(end - G)).transpose(-1, -2), E)
    return o, E, S


def _plain_rule(d):
    c = d["case"]
    H, gate, squash = c["H"], c["gate"], c["precond"] == "squash"
    C = min(_C, d["T"])
    take, at, live = _padded(d, C)
    group = H // c["Hk"]
    tok = {n: take(d[n], group if n in "qk" else 1) for n in ("q", "k", "v", "beta", "g", "beta_p", "g_p")}
    tok = {n: None if x is None else x.transpose(1, 2) for n, x in tok.items()}   # [N, H, T, ...]
    src, dst = d["slots"].long(), d["slots_out"].long()
    S = d["S"][src]
    A = d["A"][src] if squash else None
    if d["fresh"] is not None:
        keep = (d["fresh"] == 0).float()
        S = S * keep[:, None, None, None]
        A = A * keep[:, None, None] if squash else None
    if c["kind"] == "draft":
        S, A = _plain_commit(d, S, A)
    N, T = live.shape
    G0 = torch.zeros(N, H, T, 1, device=S.device)
    os, S1 = [], S
    for i in range(0, T, C):   # the chunks of a sequence, one after the other
        x = {n: None if y is None else y[:, :, i:i + C] for n, y in tok.items()}
        kt, At = x["k"], None
        if squash:
            kt, At = _write_keys(x["k"], x["beta_p"], x["g_p"], d["log_a_scale"], A)
        g = G0[:, :, i:i + C] if gate == "none" else x["g"][..., None] if gate == "scalar" else x["g"]
        G = torch.cumsum(g, 2)
        o, E, S1 = _plain_chunk(x["q"], x["k"], kt, x["v"], x["beta"], G, S1)
        if squash and c["kind"] != "draft":
            A = At[:, :, -1]
        os.append(o)
    o = torch.empty(d["v"].shape, device=S.device, dtype=d["v"].dtype)
    o[at[live]] = torch.cat(os, 2).transpose(1, 2)[live].to(o.dtype)
    if c["kind"] == "draft":   # the state stays; the tokens' rows are left pending
        rec = [kt, E, G if gate == "channel" else G.expand(-1, -1, -1, 4)] + ([At] if squash else [])
        rec = torch.cat(rec, -1).transpose(1, 2)
        d["tape"][dst] = torch.where(live[:, :, None, None], rec, d["tape"][dst])
        d["pending"][dst] = live.sum(1)[:, None].to(torch.int32)
    d["S"][dst] = S if c["kind"] == "draft" else S1
    if squash:
        d["A"][dst] = A
    return _outputs(d, o)


def _plain_commit(d, S, A):
    """The accepted tokens of the last round, applied to the states."""
    c = d["case"]
    src = d["slots"].long()
    n = torch.minimum(d["accepted"].long(), d["pending"][src, 0].long())
    tape = d["tape"][src].transpose(1, 2)   # [N, H, T, record]
    n_g = c["dk"] if c["gate"] == "channel" else 4
    kt, e, G, At = tape.split([c["dk"], c["dv"], n_g, tape.shape[-1] - c["dk"] - c["dv"] - n_g], -1)
    G = G if c["gate"] == "channel" else G[..., :1]
    at = (n - 1).clamp(min=0)[:, None, None, None]
    end = torch.gather(G, 2, at.expand(-1, G.shape[1], 1, G.shape[3]))
    w = torch.exp((end - G).clamp(max=0.0)) * (torch.arange(tape.shape[2], device=S.device)[None, :] < n[:, None])[:, None, :, None]
    some = (n > 0)[:, None, None, None]
    S = torch.where(some, torch.exp(end).transpose(-1, -2) * S, S) + torch.matmul((kt * w).transpose(-1, -2), e)
    if A is not None:
        A = torch.where(some[..., 0], torch.gather(At, 2, at.expand(-1, At.shape[1], 1, At.shape[3]))[:, :, 0], A)
    return S, A


def _plain_verify(d):
    p, q, ids, starts = d["p"], d["q"], d["ids"].long(), d["starts"].long()
    first, rows = starts[:-1], starts[1:] - starts[:-1]
    t = torch.arange(d["case"]["K"], device=ids.device)[None, :]
    live = t + 1 < rows[:, None]                        # draft t + 1 of the sequence
    at = torch.where(live, first[:, None] + t, 0)
    nxt = torch.where(live, at + 1, 0)
    x = ids[nxt]
    px = p[at, x].double()
    qx = q[nxt, x].double() if q is not None else torch.ones_like(px)
    held = live & (d["u"][at].double() * qx < px)
    n = torch.cumprod(held.long(), 1).sum(1)            # drafts that hold
    row = first + n
    w = p[row].double()
    refused = n + 1 < rows
    after = torch.where(refused, row + 1, 0)
    if q is not None:
        rest = (w - q[after].double()).clamp(min=0.0)
    else:
        rest = w.clone()
        rest.scatter_(1, ids[after][:, None], 0.0)
    w = torch.where((refused & (rest.sum(1) > 0))[:, None], rest, w)
    cum = torch.cumsum(w, 1)
    token = (cum <= (d["r"].double() * cum[:, -1])[:, None]).sum(1)
    return {"accepted": (n + 1).to(torch.int32), "token": token.to(torch.int32)}


def work(case):
    c = case
    if c["kind"] == "verify":
        # of each sequence the row it stops at, and where a draft was refused (about two in three) the drafting model's too
        rows = c["N"] * c["V"] * (4 if c["io"] == "f32" else 2)
        return {"bytes": rows * (5 / 3 if c["q"] else 1), "flops": rows / 2}
    N, H, Hk, dk, dv = (c[n] for n in ("N", "H", "Hk", "dk", "dv"))
    tokens = sum(_lengths(c))
    esz = 2 if c["io"] == "bf16" else 4
    squash = c["precond"] == "squash"
    n_g = {"none": 0, "scalar": 1, "channel": dk}[c["gate"]]
    state = 4 * H * (dk * dv + (dk if squash else 0))
    token = esz * (2 * Hk * dk + 2 * H * dv) + 4 * H * (1 + n_g + (2 if squash else 0))
    flops = tokens * H * 6 * dk * dv
    reads = N * (0.5 if c["kind"] == "prefill" else 1)   # half the prompts are new
    total = (N + reads) * state + tokens * token
    if c["kind"] == "draft":
        # the records: the accepted half is read, the new ones are written
        total += 1.5 * tokens * 4 * H * (dk + dv + n_g + (dk if squash else 0))
        flops += 0.5 * tokens * H * 2 * dk * dv
    return {"bytes": total, "flops": flops}


# ---------------------------------------------------------------- in 64 bits
def exact(case, seed):
    """The definitions, in 64 bits: the rule token after token, the verification draft after draft."""
    d = prepare(case, seed)
    return _exact_verify(d) if case["kind"] == "verify" else _exact_rule(d)


def _exact_rule(d):
    c = d["case"]
    N, T, H, dk, dv = c["N"], c["T"], c["H"], c["dk"], c["dv"]
    S_all, A_all = d["S"].double(), None if d["A"] is None else d["A"].double()
    src, dst, starts = d["slots"].long(), d["slots_out"].long(), d["starts"].long()
    S, A = S_all[src], None if A_all is None else A_all[src]
    tape, pending = (d["tape"].double(), d["pending"]) if c["kind"] == "draft" else (None, None)
    for n in range(N):
        if d["fresh"] is not None and int(d["fresh"][n]):
            S[n] = 0
            if A is not None:
                A[n] = 0
        if tape is not None:
            rec, m = tape[src[n]], min(int(d["accepted"][n]), int(pending[src[n], 0]))
            before = None
            for s in range(m):
                Gs = rec[s, :, dk + dv:dk + dv + (dk if c["gate"] == "channel" else 1)]
                a = torch.exp(Gs if before is None else Gs - before)      # this token's decay
                before = Gs
                S[n] = a[:, :, None] * S[n] + rec[s, :, :dk, None] * rec[s, :, None, dk:dk + dv]
                if A is not None:
                    A[n] = rec[s, :, -dk:]
    S_kept, A_kept = S.clone(), None if A is None else A.clone()
    o = torch.zeros(d["v"].shape, dtype=_F64, device="cuda")
    G = torch.zeros(N, H, dk, dtype=_F64, device="cuda")
    group = H // c["Hk"]
    for t in range(T):
        n = (starts[1:] - starts[:-1] > t).nonzero()[:, 0]
        i = starts[n] + t
        q, k, v = (d[x][i].double() for x in "qkv")
        q, k = q.repeat_interleave(group, 1), k.repeat_interleave(group, 1)
        b = d["beta"][i].double()
        kt = k
        if A is not None:
            An = torch.exp(d["g_p"][i].double())[..., None] * A[n] + d["beta_p"][i].double()[..., None] * k * k
            r = torch.log(An) - torch.exp(d["log_a_scale"].double())[None, :, None]
            kt = k * torch.exp(-math.log(_X) * r / (1 + r.abs()))
            A[n] = An
        Sn = S[n]
        if d["g"] is not None:
            g = d["g"][i].double()
            g = g if g.dim() == 3 else g[..., None].expand(-1, -1, dk)
            G[n] = G[n] + g
            Sn = torch.exp(g)[..., None] * Sn
        e = b[..., None] * (v - (k[..., None] * Sn).sum(2))
        Sn = Sn + kt[..., None] * e[:, :, None]
        o[i] = (q[..., None] * Sn).sum(2)
        S[n] = Sn
        if tape is not None:
            tape[dst[n], t] = torch.cat([kt, e, G[n] if c["gate"] == "channel" else G[n][..., :4]] + ([A[n]] if A is not None else []), -1)
    S_all[dst] = S_kept if tape is not None else S
    if A is not None:
        A_all[dst] = A_kept if tape is not None else A
    out = {"o": o, "S": S_all, "A": A_all}
    if tape is not None:
        pending = pending.clone()
        pending[dst] = (starts[1:] - starts[:-1])[:, None].to(torch.int32)
        out.update(tape=tape, pending=pending)
    return {n: x for n, x in out.items() if x is not None}


def _exact_verify(d):
    starts = d["starts"].tolist()
    ids, u, r = d["ids"].tolist(), d["u"].double().tolist(), d["r"].double().tolist()
    accepted, token = [], []
    for n, (lo, hi) in enumerate(zip(starts, starts[1:])):
        row = lo
        while row + 1 < hi:
            x = ids[row + 1]
            if not u[row] * (float(d["q"][row + 1, x]) if d["q"] is not None else 1.0) < float(d["p"][row, x]):
                break
            row += 1
        w = d["p"][row].double().cpu()
        if row + 1 < hi:
            less = torch.zeros_like(w)
            less[ids[row + 1]] = math.inf
            if d["q"] is not None:
                less = d["q"][row + 1].double().cpu()
            rest = torch.relu(w - less)
            w = rest if rest.sum() > 0 else w
        w = w.numpy().cumsum()
        accepted.append(row - lo + 1)
        token.append(int(w.searchsorted(r[n] * w[-1], side="right")))
    make = dict(dtype=torch.int32, device="cuda")
    return {"accepted": torch.tensor(accepted, **make), "token": torch.tensor(token, **make)}
