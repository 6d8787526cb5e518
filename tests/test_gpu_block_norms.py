"""The norms around the rule on the GPU: pdn_residual_norm, pdn_head_norm and their backward
passes against their definitions in 64 bits (bounds in block_util)."""
import numpy as np
import pytest

import block_util as bu
from block_util import ONE, TWO, close, dtype, seen

pytestmark = pytest.mark.gpu
EPS = 1e-5


def put(x, io, off=0):
    """To the device, `off` elements into an allocation."""
    import torch
    if x is None:
        return None
    t = torch.from_numpy(np.ascontiguousarray(x)).to(dtype(io))
    room = torch.empty(t.numel() + off + 8, dtype=t.dtype, device="cuda")
    v = room[off:off + t.numel()].view(t.shape)
    v.copy_(t)
    return v


def rnorm_inputs(rng, rows, D, io, st, post, scale, residual, weight):
    f = lambda *s: rng.standard_normal(s)   # noqa: E731
    v = lambda on, *s: seen(1 + 0.3 * f(*s), "f32") if on else None   # noqa: E731
    d = dict(y=seen(f(rows, D) * np.exp(f(D)), io), residual=seen(2 * f(rows, D), st) if residual else None,
             weight=v(weight, D), post_weight=v(post == "weight", D), scale=v(scale, D))
    return d, dict(post=bool(post), alpha=float(np.float32(0.7)), eps=float(np.float32(EPS)))


ROWS = [(1, 1), (3, 7), (2, 64), (5, 513), (17, 1001), (4, 2048), (3, 4104), (2, 8192), (2, 8201), (2, 16384), (70, 128)]
MODES = [("bf16", "bf16", "", False, True, True), ("bf16", "f32", "weight", True, True, True), ("f32", "f32", "", True, False, True),
         ("f32", "bf16", "ones", False, True, False), ("f32", "f32", "weight", False, True, True), ("bf16", "bf16", "weight", True, False, False)]


@pytest.mark.parametrize("rows,D", ROWS)
@pytest.mark.parametrize("io,st,post,scale,residual,weight", MODES)
def test_residual_norm(rows, D, io, st, post, scale, residual, weight):
    import paper_2604_21100_amd as pdn
    d, kw = rnorm_inputs(np.random.default_rng(rows + D), rows, D, io, st, post, scale, residual, weight)
    want = bu.rnorm(d["y"], d["residual"], d["weight"], kw["post"], d["post_weight"], d["scale"], kw["alpha"], kw["eps"])
    for off in (0, 1):   # (aligned to 16 bytes, and to an element only)
        vec = {n: put(d[n], "f32", off) for n in ("weight", "post_weight", "scale")}
        u, h = pdn.pdn_residual_norm(put(d["y"], io, off), put(d["residual"], st, off), post_norm=kw["post"], alpha=kw["alpha"], eps=EPS,
                                     h_dtype=dtype(st), **vec)
        assert u.dtype == dtype(io) and h.dtype == dtype(st)
        close(h, *want[1], st, ONE, "h")
        close(u, *want[0], io, ONE, "u")


@pytest.mark.parametrize("rows,D", ROWS + [(2500, 33)])
@pytest.mark.parametrize("io,st,post,scale,residual,weight", MODES)
def test_residual_norm_bwd(rows, D, io, st, post, scale, residual, weight):
    import paper_2604_21100_amd as pdn
    rng = np.random.default_rng(rows + 3 * D)
    d, kw = rnorm_inputs(rng, rows, D, io, st, post, scale, True, weight)
    h, du = d.pop("residual"), seen(rng.standard_normal((rows, D)), io)
    dh = seen(rng.standard_normal((rows, D)), st) if residual else None
    y = d["y"] if post or scale else None
    want = bu.rnorm_bwd(du, dh, h, y, d["weight"], kw["post"], d["post_weight"], d["scale"], kw["alpha"], kw["eps"])
    for off in (0, 1):
        vec = {n: put(d[n], "f32", off) for n in ("weight", "post_weight", "scale")}
        got = pdn.pdn_residual_norm_bwd(put(du, io, off), put(h, st, off), put(y, io, off), dh=put(dh, st, off), post_norm=kw["post"],
                                        alpha=kw["alpha"], eps=EPS, **vec)
        names = {"dy", "dresidual"} | {"d" + n for n in vec if vec[n] is not None}
        assert set(got) == names
        for n in names:
            kind = {"dy": io, "dresidual": st}.get(n, "f32")
            close(got[n], *want[n], kind, TWO if post else ONE, n)


def test_residual_norm_more_rows_than_workgroups():
    import torch
    import paper_2604_21100_amd as pdn
    rows = (1 << 20) + 5
    y = torch.randn(rows, 4, device="cuda")
    u, h = pdn.pdn_residual_norm(y, eps=EPS)
    assert torch.equal(h, y)
    d = y.double()
    want = d / (d.square().mean(1, keepdim=True) + EPS).sqrt()
    assert ((u.double() - want).abs() <= 64 * bu.U * want.abs()).all()


def test_residual_norm_in_place_and_parts_left_out():
    """h is residual itself, dresidual dh itself; h, dresidual, vectors' gradients not wanted; no rows."""
    import torch
    import paper_2604_21100_amd as pdn
    g = torch.Generator(device="cuda").manual_seed(1)
    r = lambda *s: torch.randn(s, generator=g, device="cuda")   # noqa: E731
    y, x, w = r(2, 9, 300).bfloat16(), r(2, 9, 300), r(300)
    u, h = pdn.pdn_residual_norm(y, x, weight=w, alpha=0.5)
    x1 = x.clone()
    u1, h1 = pdn.pdn_residual_norm(y, x1, weight=w, alpha=0.5, h=x1)
    assert h1 is x1 and torch.equal(h1, h) and torch.equal(u, u1)
    u2, none = pdn.pdn_residual_norm(y, x, weight=w, alpha=0.5, want_h=False, u=torch.empty_like(u))
    assert none is None and torch.equal(u2, u)
    du, dh = r(2, 9, 300).bfloat16(), r(2, 9, 300)
    a = pdn.pdn_residual_norm_bwd(du, h, dh=dh, weight=w, alpha=0.5)
    d1 = dh.clone()
    b = pdn.pdn_residual_norm_bwd(du, h, dh=d1, weight=w, alpha=0.5, outputs=dict(dresidual=d1))
    assert b["dresidual"] is d1 and all(torch.equal(a[n], b[n]) for n in a)
    c = pdn.pdn_residual_norm_bwd(du, h, dh=dh, weight=w, alpha=0.5, want_residual=False, want_vectors=False)
    assert set(c) == {"dy"} and torch.equal(c["dy"], a["dy"])
    none = torch.empty(0, 300, device="cuda")
    e = pdn.pdn_residual_norm_bwd(none, none, none, weight=w, scale=w, post_norm=True, post_weight=w)
    for n in ("dweight", "dscale", "dpost_weight"):
        assert torch.equal(e[n], torch.zeros(300, device="cuda"))
    assert pdn.pdn_residual_norm(none, none)[0].shape == (0, 300)


def test_rows_do_not_meet():
    """NaN and infinities show in their own rows (and channels' sums), zero rows give zeros."""
    import torch
    import paper_2604_21100_amd as pdn
    torch.manual_seed(2)
    y, x, w = torch.randn(5, 200, device="cuda"), torch.randn(5, 200, device="cuda"), torch.randn(200, device="cuda")
    u, h = pdn.pdn_residual_norm(y, x, weight=w, post_norm=True, scale=w)
    bad = y.clone()
    bad[1, 7], bad[3, 0] = float("nan"), float("inf")
    u1, h1 = pdn.pdn_residual_norm(bad, x, weight=w, post_norm=True, scale=w)
    for t, t1 in ((u, u1), (h, h1)):
        assert torch.equal(t[[0, 2, 4]], t1[[0, 2, 4]])
        assert t1[1].isnan().all() and t1[3, 0].isnan()
    zero = torch.zeros(2, 200, device="cuda")
    u, h = pdn.pdn_residual_norm(zero, zero, weight=w, post_norm=True)
    assert torch.equal(u, zero) and torch.equal(h, zero)
    g = pdn.pdn_residual_norm_bwd(torch.ones_like(zero), zero, zero, weight=w, post_norm=True, post_weight=w, eps=1e-30)
    assert all(t.isfinite().all() for t in g.values())
    x = torch.randn(4, 3, 40, device="cuda")
    z = torch.randn(4, 3, 40, device="cuda")
    a = pdn.pdn_head_norm(x, z=z)
    b = x.clone()
    b[2, 1, 5] = float("nan")
    b = pdn.pdn_head_norm(b, z=z)
    assert b[2, 1].isnan().all()
    b[2, 1] = a[2, 1]
    assert torch.equal(a, b)
    g = pdn.pdn_head_norm_bwd(torch.ones_like(x), torch.zeros_like(x), norm="l2", eps=1e-30)
    assert g["dx"].isfinite().all()


def test_gates_of_any_size():
    """The gate at both ends of its range, infinities too."""
    import torch
    import paper_2604_21100_amd as pdn
    inf = float("inf")
    for dt in (torch.float32, torch.bfloat16):
        z = torch.tensor([-inf, -1e30, -300.0, -100.0, -20.0, 0.0, 20.0, 100.0, 1e30, inf], device="cuda").to(dt).view(1, 1, 10)
        x = torch.ones(1, 1, 10, device="cuda", dtype=dt)
        y = pdn.pdn_head_norm(x, z=z, act="sigmoid", eps=1e-12)
        assert torch.allclose(y.float(), torch.sigmoid(z.float()), rtol=2 ** -7, atol=1e-38)
        y = pdn.pdn_head_norm(x[..., 1:9].contiguous(), z=z[..., 1:9].contiguous(), eps=1e-12)
        s = torch.nn.functional.silu(z[..., 1:9].float())
        assert y.isfinite().all() and torch.allclose(y.float(), s, rtol=2 ** -7, atol=1e-36)


HEADS = [(1, 1, 1), (3, 2, 33), (64, 3, 64), (37, 5, 128), (1000, 2, 128), (9, 4, 200), (5, 3, 512), (2500, 1, 8), (300, 12, 16)]
KINDS = [("bf16", "rms", "shared", "silu"), ("f32", "rms", "head", "sigmoid"), ("bf16", "l2", "", "none"), ("f32", "l2", "shared", "none"),
         ("bf16", "rms", "head", "none"), ("f32", "rms", "", "silu"), ("bf16", "l2", "shared", "sigmoid")]


def head_case(rng, M, H, d, io, norm, weight, act):
    f = lambda *s: rng.standard_normal(s)   # noqa: E731
    w = {"": None, "shared": (d,), "head": (H, d)}[weight]
    return dict(x=seen(f(M, H, d) * np.exp(f(M, H, 1)), io), dy=seen(f(M, H, d), io), z=None if act == "none" else seen(3 * f(M, H, d), io),
                weight=None if w is None else seen(1 + 0.3 * f(*w), "f32"))


def as_slice(x, io, pad):
    """The heads as a slice of wider rows, `pad` elements in."""
    import torch
    if x is None:
        return None
    M, H, d = x.shape
    wide = torch.full((M, H * d + 2 * pad + 1), float("nan"), dtype=dtype(io), device="cuda")
    v = wide[:, pad:pad + H * d].view(M, H, d)
    v.copy_(torch.from_numpy(x).to(dtype(io)))
    return v


@pytest.mark.parametrize("M,H,d", HEADS)
@pytest.mark.parametrize("io,norm,weight,act", KINDS)
def test_head_norm(M, H, d, io, norm, weight, act):
    import paper_2604_21100_amd as pdn
    c = head_case(np.random.default_rng(M + H * d), M, H, d, io, norm, weight, act)
    kw = dict(norm=norm, act=act, eps=EPS, weight=put(c["weight"], "f32"))
    e = float(np.float32(EPS))
    want = bu.hnorm(c["x"], norm, c["weight"], c["z"], act, e)
    back = bu.hnorm_bwd(c["dy"], c["x"], norm, c["weight"], c["z"], act, e)
    for pad in (None, 0, 16, 3):
        to = (lambda n: put(c[n], io)) if pad is None else (lambda n: as_slice(c[n], io, pad))   # noqa: B023
        close(pdn.pdn_head_norm(to("x"), z=to("z"), **kw), *want, io, ONE, "y")
        got = pdn.pdn_head_norm_bwd(to("dy"), to("x"), z=to("z"), **kw)
        assert set(got) == {"dx"} | ({"dz"} if c["z"] is not None else set()) | ({"dweight"} if weight else set())
        for n, t in got.items():
            close(t, *back[n], "f32" if n == "dweight" else io, ONE, n)


def test_head_norm_in_place_and_in_one_projection():
    """y is x itself, dx dy itself; gradients written into the slices of one projection's; batched tokens."""
    import torch
    import paper_2604_21100_amd as pdn
    torch.manual_seed(3)
    B, T, H, d = 2, 21, 4, 64
    proj = torch.randn(B, T, 3 * H * d, device="cuda").bfloat16()
    x, z, v = (t.unflatten(-1, (H, d)) for t in proj.split(H * d, -1))
    w = torch.randn(H, d, device="cuda")
    y = pdn.pdn_head_norm(x, weight=w, z=z)
    assert y.shape == (B, T, H, d) and y.is_contiguous()
    dy = torch.randn_like(y)
    g = pdn.pdn_head_norm_bwd(dy, x, weight=w, z=z)
    dproj = torch.full_like(proj, 7.0)
    dx, dz, dv = (t.unflatten(-1, (H, d)) for t in dproj.split(H * d, -1))
    g1 = pdn.pdn_head_norm_bwd(dy, x, weight=w, z=z, outputs=dict(dx=dx, dz=dz))
    assert g1["dx"] is dx and torch.equal(dx, g["dx"]) and torch.equal(dz, g["dz"]) and torch.equal(g1["dweight"], g["dweight"])
    assert (dv == 7.0).all()
    dy1 = dy.clone()
    g2 = pdn.pdn_head_norm_bwd(dy1, x, weight=w, z=z, outputs=dict(dx=dy1), want_vectors=False)
    assert torch.equal(dy1, g["dx"]) and set(g2) == {"dx", "dz"}
    kept = proj.clone()
    out = pdn.pdn_head_norm(x, weight=w, z=z, y=x)
    assert out is x and torch.equal(x, y) and torch.equal(proj[..., H * d:], kept[..., H * d:])
    e = pdn.pdn_head_norm_bwd(dy[:0], x[:0], weight=w, z=z[:0])
    assert torch.equal(e["dweight"], torch.zeros_like(w)) and e["dx"].shape[0] == 0


def test_many_heads():
    """More heads than parts: a workgroup a head."""
    import torch
    import paper_2604_21100_amd as pdn
    torch.manual_seed(4)
    M, H, d = 2, 5000, 16
    x, dy, w = torch.randn(M, H, d, device="cuda"), torch.randn(M, H, d, device="cuda"), torch.rand(H, d, device="cuda")
    c = dict(x=x.cpu().double().numpy(), dy=dy.cpu().double().numpy(), w=w.cpu().double().numpy())
    e = float(np.float32(EPS))
    close(pdn.pdn_head_norm(x, weight=w, eps=EPS), *bu.hnorm(c["x"], "rms", c["w"], None, "none", e), "f32", ONE)
    for weight, cw in ((w, c["w"]), (w[0].contiguous(), c["w"][0])):
        got, want = pdn.pdn_head_norm_bwd(dy, x, weight=weight, eps=EPS), bu.hnorm_bwd(c["dy"], c["x"], "rms", cw, None, "none", e)
        for n in got:
            close(got[n], *want[n], "f32", ONE, n)


def test_same_bits_streams_and_graphs():
    """Twice the same bits; on another stream; two graphs with workspaces of their own, replayed in turn with eager
    calls between."""
    import torch
    import paper_2604_21100_amd as pdn
    torch.manual_seed(5)
    R, D, H, d = 3000, 640, 5, 128
    r = lambda *s: torch.randn(s, device="cuda")   # noqa: E731
    y, x, du, dh, w, s = r(R, D).bfloat16(), r(R, D), r(R, D).bfloat16(), r(R, D), r(D), r(D)

    def step(outs=None, ws=(None, None)):
        o = outs or {}
        u, h = pdn.pdn_residual_norm(y, x, weight=w, post_norm=True, post_weight=s, scale=s, u=o.get("u"), h=o.get("h"))
        a = pdn.pdn_residual_norm_bwd(du, h, y, dh=dh, weight=w, post_norm=True, post_weight=s, scale=s, outputs=o.get("a"), workspace=ws[0])
        n = pdn.pdn_head_norm(u.view(R, H, d), z=y.view(R, H, d), y=o.get("n"))
        b = pdn.pdn_head_norm_bwd(n, u.view(R, H, d), z=y.view(R, H, d), weight=w[:d].contiguous() if outs is None else o["w"],
                                  outputs=o.get("b"), workspace=ws[1])
        return [u, h, n] + [a[k] for k in sorted(a)] + [b[k] for k in sorted(b)]

    first = step()
    for p, q in zip(first, step()):
        assert torch.equal(p, q)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    u, _ = pdn.pdn_residual_norm(y, x, weight=w, post_norm=True, post_weight=s, scale=s, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(u, first[0])

    def buffers():
        e = torch.empty_like
        a = dict(dy=e(y), dresidual=e(x), dweight=e(w), dpost_weight=e(w), dscale=e(w))
        b = dict(dx=e(y).view(R, H, d), dz=e(y).view(R, H, d), dweight=torch.empty(d, device="cuda"))
        return dict(u=e(y), h=e(x), n=e(y).view(R, H, d), a=a, b=b, w=w[:d].contiguous())

    graphs = []
    for _ in range(2):
        outs = buffers()
        ws = tuple(torch.empty(1 << 25, dtype=torch.uint8, device="cuda") for _ in range(2))
        got = step(outs, ws)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            got = step(outs, ws)
        graphs.append((g, got, ws))
    for turn in range(3):
        for g, got, _ in graphs:
            for t in got:
                t.fill_(float("nan"))
            g.replay()
            eager = step()
            torch.cuda.synchronize()
            for p, q, e in zip(first, got, eager):
                assert torch.equal(p, q) and torch.equal(p, e)


@pytest.mark.parametrize("rows,D", [(5000, 24), (3300, 300), (1700, 520), (900, 1400), (530, 2056), (520, 3001), (300, 5000), (270, 9000)])
@pytest.mark.parametrize("io,st", [("bf16", "f32"), ("f32", "f32")])
def test_backward_over_more_rows_than_parts(rows, D, io, st):
    """Each width's form with several rows a part: every vector's gradient."""
    import paper_2604_21100_amd as pdn
    rng = np.random.default_rng(rows)
    d, kw = rnorm_inputs(rng, rows, D, io, st, "weight", True, True, True)
    h, du, dh = d.pop("residual"), seen(rng.standard_normal((rows, D)), io), seen(rng.standard_normal((rows, D)), st)
    want = bu.rnorm_bwd(du, dh, h, d["y"], d["weight"], True, d["post_weight"], d["scale"], kw["alpha"], kw["eps"])
    got = pdn.pdn_residual_norm_bwd(put(du, io), put(h, st), put(d["y"], io), dh=put(dh, st), post_norm=True, alpha=kw["alpha"], eps=EPS,
                                    **{n: put(d[n], "f32") for n in ("weight", "post_weight", "scale")})
    for n in want:
        close(got[n], *want[n], {"dy": io, "dresidual": st}.get(n, "f32"), TWO, n)


def test_offsets_past_32_bits():
    """The last rows of tensors of more than 2^31 elements: the bits of a small call."""
    import torch
    import paper_2604_21100_amd as pdn
    g = torch.Generator(device="cuda").manual_seed(7)
    R, D, H, n = 1_060_000, 2048, 16, 3
    r = lambda *s: torch.randn(s, generator=g, device="cuda")   # noqa: E731
    w = r(D)
    y, x, du = (torch.zeros(R, D, dtype=torch.bfloat16, device="cuda") for _ in range(3))
    for t in (y, x, du):
        t[-n:] = r(n, D)
    kw = dict(weight=w, post_norm=True, scale=w)
    u, h = pdn.pdn_residual_norm(y, x, **kw)
    us, hs = pdn.pdn_residual_norm(y[-n:], x[-n:], **kw)
    assert torch.equal(u[-n:], us) and torch.equal(h[-n:], hs) and not u[:-n].any() and not h[:-n].any()
    a, b = pdn.pdn_residual_norm_bwd(du, h, y, **kw), pdn.pdn_residual_norm_bwd(du[-n:], hs, y[-n:], **kw)
    for m in ("dy", "dresidual"):
        assert torch.equal(a[m][-n:], b[m]) and not a[m][:-n].any()
    heads = lambda t: t.view(-1, H, D // H)   # noqa: E731
    del a
    o, os = pdn.pdn_head_norm(heads(x), z=heads(y)), pdn.pdn_head_norm(heads(x[-n:]), z=heads(y[-n:]))
    assert torch.equal(o[-n:], os) and not o[:-n].any()
    del o
    a, b = pdn.pdn_head_norm_bwd(heads(du), heads(x), z=heads(y)), pdn.pdn_head_norm_bwd(heads(du[-n:]), heads(x[-n:]), z=heads(y[-n:]))
    for m in a:
        assert torch.equal(a[m][-n:], b[m]) and not a[m][:-n].any()


@pytest.mark.parametrize("D", [5, 300, 1000, 1001, 4104, 9001])
def test_in_place_at_every_width(D):
    """h in residual's place and dresidual in dh's, in each form of a row: the bits of the calls that do not."""
    import torch
    import paper_2604_21100_amd as pdn
    torch.manual_seed(D)
    R = 700
    y, x, du, dh = (torch.randn(R, D, device="cuda") for _ in range(4))
    w = torch.randn(D, device="cuda")
    kw = dict(weight=w, post_norm=True, post_weight=w, scale=w)
    u, h = pdn.pdn_residual_norm(y, x, **kw)
    a = pdn.pdn_residual_norm_bwd(du, h, y, dh=dh, **kw)
    u1, h1 = pdn.pdn_residual_norm(y, x, h=x, **kw)
    assert h1 is x and torch.equal(h, x) and torch.equal(u, u1)
    b = pdn.pdn_residual_norm_bwd(du, h, y, dh=dh, outputs=dict(dresidual=dh), **kw)
    assert b["dresidual"] is dh and all(torch.equal(a[n], b[n]) for n in a)


@pytest.mark.parametrize("d", [5, 8, 33, 128, 200])
@pytest.mark.parametrize("each", [False, True])
def test_head_norm_in_place_at_every_width(d, each):
    import torch
    import paper_2604_21100_amd as pdn
    torch.manual_seed(d)
    M, H = 900, 6
    x, z, dy = (torch.randn(M, H, d, device="cuda").bfloat16() for _ in range(3))
    w = torch.randn(H, d, device="cuda") if each else torch.randn(d, device="cuda")
    y, g = pdn.pdn_head_norm(x, weight=w, z=z), pdn.pdn_head_norm_bwd(dy, x, weight=w, z=z)
    b = pdn.pdn_head_norm_bwd(dy, x, weight=w, z=z, outputs=dict(dx=dy))
    assert b["dx"] is dy and all(torch.equal(g[n], b[n]) for n in g)
    assert pdn.pdn_head_norm(x, weight=w, z=z, y=x) is x and torch.equal(x, y)
