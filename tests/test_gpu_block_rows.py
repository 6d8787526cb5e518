"""The norms around the rule over many rows: each width's form with several rows a workgroup, against the definitions in
64 bits (on the device, as the tensors are large), with the bounds of block_util: a lane adds up at most 64
rows' terms of a vector's gradient in fp32, its neighbours' 8 times more, so ONE = 128 and TWO = 320 roundings hold
them with the factor's 24."""
import pytest

from block_util import HALF, ONE, TWO, dtype

pytestmark = pytest.mark.gpu
EPS = 1e-5


def close(got, want, mag, io, bound, name):
    off, room = (got.double() - want).abs(), HALF[io] * want.abs() + bound * mag * (1 + HALF[io])
    assert got.isfinite().all() and (off <= room).all(), (name, (off / room.clamp(min=1e-300)).max().item())


def factor(x, width):
    return (x.square().sum(-1, keepdim=True) / width + EPS).rsqrt()


def pull(x, g, mg, width):
    """The gradient of x where x times its factor is the norm and g the norm's gradient, of magnitude mg."""
    r = factor(x, width)
    n = x * r
    return r * (g - n * (g * n).sum(-1, keepdim=True) / width), r * (mg + n.abs() * (mg * n.abs()).sum(-1, keepdim=True) / width)


def summed(x, dims):
    return x.sum(dims), x.abs().sum(dims)


# rows so that each workgroup takes five or more: as many parts as compute units hold, rows of 513 columns on one each, below
# several at once
WIDTHS = [(250_000, 24), (130_000, 33), (15_500, 300), (15_500, 509), (5_200, 1400), (5_200, 1403), (2_700, 3000), (2_700, 3001), (1_400, 5000),
          (1_400, 5003), (1_300, 9000), (1_300, 9001)]
PARTS = [(False, False, False), (False, False, True), (True, False, True), (False, True, True), (True, True, False), (True, True, True)]


@pytest.mark.parametrize("rows,D", WIDTHS)
@pytest.mark.parametrize("io,st", [("bf16", "bf16"), ("f32", "f32"), ("bf16", "f32")])
def test_residual_norm_backward(rows, D, io, st):
    import torch
    import paper_2604_21100_amd as pdn
    g = torch.Generator(device="cuda").manual_seed(D)
    r = lambda *s: torch.randn(s, generator=g, device="cuda")   # noqa: E731
    y, du, h, dh0 = r(rows, D).to(dtype(io)), r(rows, D).to(dtype(io)), r(rows, D).to(dtype(st)), r(rows, D).to(dtype(st))
    w, wp, s = 1 + 0.3 * r(D), 1 + 0.3 * r(D), 1 + 0.3 * r(D)
    alpha = 0.75
    for post, scale, with_dh in PARTS:
        dh = dh0 if with_dh else None
        got = pdn.pdn_residual_norm_bwd(du, h, y if post or scale else None, dh=dh, weight=w, post_norm=post, post_weight=wp if post else None,
                                        scale=s if scale else None, alpha=alpha, eps=EPS)
        x, a, gu = h.double(), y.double(), du.double() * w.double()
        t, mt = pull(x, gu, gu.abs(), D)
        if with_dh:
            t, mt = t + dh.double(), mt + dh.double().abs()
        bound = TWO if post else ONE
        close(got["dresidual"], t, mt, st, bound, "dresidual")
        close(got["dweight"], *summed(du.double() * x * factor(x, D), 0), "f32", bound, "dweight")
        n = a * factor(a, D) if post else a
        b, mb = alpha * t, alpha * mt
        if scale:
            m = n * wp.double() if post else n
            close(got["dscale"], (b * m).sum(0), (mb * m.abs()).sum(0), "f32", bound, "dscale")
            b, mb = b * s.double(), mb * s.double().abs()
        if post:
            close(got["dpost_weight"], (b * n).sum(0), (mb * n.abs()).sum(0), "f32", bound, "dpost_weight")
            b, mb = pull(a, b * wp.double(), mb * wp.double().abs(), D)
        close(got["dy"], b, mb, io, bound, "dy")
        assert set(got) == {"dy", "dresidual", "dweight"} | ({"dscale"} if scale else set()) | ({"dpost_weight"} if post else set())


# (heads that divide neither the groups of a workgroup nor those of all, so that a group's head changes from row to row)
HEADS = [(8000, 5, 128), (4000, 12, 200), (30011, 3, 33), (16001, 13, 300), (150_000, 7, 5), (9001, 5, 512)]


@pytest.mark.parametrize("M,H,d", HEADS)
@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("act", ["none", "silu", "sigmoid"])
def test_head_norm_backward(M, H, d, io, act):
    import torch
    import paper_2604_21100_amd as pdn
    g = torch.Generator(device="cuda").manual_seed(M)
    r = lambda *s: torch.randn(s, generator=g, device="cuda")   # noqa: E731
    x, dy, z = r(M, H, d).to(dtype(io)), r(M, H, d).to(dtype(io)), 3 * r(M, H, d)
    z = None if act == "none" else z.to(dtype(io))
    n = x.double()
    for norm, weight in (("rms", "shared"), ("l2", "head"), ("rms", "")):
        w = {"": None, "shared": 1 + 0.3 * r(d), "head": 1 + 0.3 * r(H, d)}[weight]
        got = pdn.pdn_head_norm_bwd(dy, x, norm=norm, weight=w, z=z, act=act, eps=EPS)
        width = d if norm == "rms" else 1
        a = slope = ms = 1.0
        if z is not None:
            s = torch.sigmoid(z.double())
            rest = torch.sigmoid(-z.double())
            a = z.double() * s if act == "silu" else s
            slope, ms = (s + a * rest, s + a.abs() * rest) if act == "silu" else (s * rest, s * rest)
        wd = 1.0 if w is None else w.double()
        gy = dy.double() * wd * a
        close(got["dx"], *pull(n, gy, gy.abs(), width), io, ONE, "dx")
        unit = n * factor(n, width)
        if z is not None:
            close(got["dz"], dy.double() * wd * unit * slope, (dy.double() * wd * unit).abs() * ms, io, ONE, "dz")
        if w is not None:
            close(got["dweight"], *summed(dy.double() * unit * a, 0 if weight == "head" else (0, 1)), "f32", ONE, "dweight")
        assert set(got) == {"dx"} | ({"dz"} if z is not None else set()) | ({"dweight"} if w is not None else set())


@pytest.mark.parametrize("rows,D", [((1 << 20) + 5, 520), ((1 << 20) + 5, 521), ((1 << 28) + 3, 4)])
def test_residual_norm_past_the_largest_grid(rows, D):
    """2^20 workgroups, of one row or of 256 short ones, then each takes another: the bits of calls on parts of the rows."""
    import torch
    import paper_2604_21100_amd as pdn
    g = torch.Generator(device="cuda").manual_seed(D)
    y = torch.randn(rows, D, generator=g, device="cuda", dtype=torch.bfloat16)
    w = torch.randn(D, generator=g, device="cuda")
    kw = dict(weight=w, post_norm=True, post_weight=w, want_h=False)
    u, _ = pdn.pdn_residual_norm(y, **kw)
    half = rows // 2
    for part in (slice(0, half), slice(half, rows)):
        assert torch.equal(u[part], pdn.pdn_residual_norm(y[part], **kw)[0])


def test_head_norm_past_the_largest_grid():
    """2^20 workgroups of four rows, a row more each: its head is another."""
    import torch
    import paper_2604_21100_amd as pdn
    M, H, d = 1_400_003, 3, 512
    g = torch.Generator(device="cuda").manual_seed(8)
    x = torch.randn(M, H, d, generator=g, device="cuda", dtype=torch.bfloat16)
    for w in (torch.randn(d, generator=g, device="cuda"), torch.randn(H, d, generator=g, device="cuda")):
        y = pdn.pdn_head_norm(x, weight=w)
        half = M // 2
        for part in (slice(0, half), slice(half, M)):
            assert torch.equal(y[part], pdn.pdn_head_norm(x[part], weight=w))
        del y
