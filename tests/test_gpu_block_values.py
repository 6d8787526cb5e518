"""The norms around the rule at values where a width's form, a type or a range could show."""
import numpy as np
import pytest

from block_util import U

pytestmark = pytest.mark.gpu
INF = float("inf")


@pytest.mark.parametrize("D", [5, 24, 33, 300, 301, 1000, 1001, 1024, 2056, 5001, 9001, 9008])
def test_an_infinite_entry_of_a_vector(D):
    """post_weight or scale with one infinite entry: h is infinite in that column and finite elsewhere, and
    so u (the factor of an infinite sum is zero) NaN there and zero elsewhere, whatever the width's form.
    In the backward an infinite weight makes the row's second sum infinite, so of rows above zero the gradients are -inf in
    the other columns."""
    import torch
    import paper_2604_21100_amd as pdn
    torch.manual_seed(D)
    R = 3
    y, x, du = (torch.randn(R, D, device="cuda").abs() + 0.5 for _ in range(3))
    w = torch.rand(D, device="cuda") + 0.5
    for j in {0, min(7, D - 1), D // 2, D - 2 if D > 1 else 0, D - 1}:
        v = w.clone()
        v[j] = INF
        rest = torch.arange(D, device="cuda") != j
        for post in (False, True):
            for kw in ([dict(scale=v)] + ([dict(post_weight=v), dict(post_weight=w, scale=v)] if post else [])):
                u, h = pdn.pdn_residual_norm(y, x, post_norm=post, **kw)
                finite = pdn.pdn_residual_norm(y, x, post_norm=post, **{n: torch.where(rest, t, w) for n, t in kw.items()})[1]
                assert torch.equal(h[:, rest], finite[:, rest]) and (h[:, j] == INF).all(), (j, post, set(kw))
                assert (u[:, rest] == 0).all() and u[:, j].isnan().all(), (j, post, set(kw))
        g = pdn.pdn_residual_norm_bwd(du, x, weight=v)
        assert (g["dresidual"][:, rest] == -INF).all() and g["dresidual"][:, j].isnan().all(), j
        assert torch.equal(g["dweight"], pdn.pdn_residual_norm_bwd(du, x, weight=w)["dweight"]), j
        if D > 1:   # (the gradients that do not read the infinite entry; dy's sum over e y has it once)
            dh = torch.full_like(x, 1e6)   # (t > 0)
            g = pdn.pdn_residual_norm_bwd(du, x, y, dh=dh, post_norm=True, post_weight=v)
            f = pdn.pdn_residual_norm_bwd(du, x, y, dh=dh, post_norm=True, post_weight=w)
            assert (g["dy"][:, rest] == -INF).all() and g["dy"][:, j].isnan().all(), j
            assert torch.equal(g["dpost_weight"], f["dpost_weight"]) and torch.equal(g["dresidual"], f["dresidual"]), j


@pytest.mark.parametrize("d", [5, 24, 33, 64, 200, 201])
@pytest.mark.parametrize("gated", [False, True])
def test_an_infinite_entry_of_a_heads_weight(d, gated):
    import torch
    import paper_2604_21100_amd as pdn
    torch.manual_seed(d)
    M, H = 3, 2
    x, dy, z = (torch.rand(M, H, d, device="cuda") + 0.5 for _ in range(3))
    z = z if gated else None
    w = torch.rand(d, device="cuda") + 0.5
    for j in {0, min(7, d - 1), d // 2, d - 2, d - 1}:
        v = w.clone()
        v[j] = INF
        rest = torch.arange(d, device="cuda") != j
        y = pdn.pdn_head_norm(x, weight=v, z=z)
        assert (y[..., j] == INF).all() and torch.equal(y[..., rest], pdn.pdn_head_norm(x, weight=w, z=z)[..., rest])
        g, f = pdn.pdn_head_norm_bwd(dy, x, weight=v, z=z), pdn.pdn_head_norm_bwd(dy, x, weight=w, z=z)
        assert (g["dx"][..., rest] == -INF).all() and g["dx"][..., j].isnan().all(), j
        assert torch.equal(g["dweight"], f["dweight"]), j
        if gated:
            assert torch.equal(g["dz"][..., rest], f["dz"][..., rest]) and g["dz"][..., j].isinf().all(), j


@pytest.mark.parametrize("D", [6, 200, 1000, 2048, 5001, 9000])
@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_rows_whose_squares_leave_fp32(D, dt):
    """A row whose sum of squares passes 3.4e38: zeros in the forward, and in the backward NaN, in that
    row and in the vectors' gradients, not zeros that look like gradients.  Other rows do not see it."""
    import torch
    import paper_2604_21100_amd as pdn
    torch.manual_seed(D)
    kind = torch.bfloat16 if dt == "bf16" else torch.float32
    R, at = 4, 2
    ok = [0, 1, 3]
    y, h, du, dh = (torch.randn(R, D, device="cuda").to(kind) for _ in range(4))
    w = torch.rand(D, device="cuda") + 0.5
    big = torch.full((D,), 1e19, device="cuda").to(kind)   # (squares of 1e38, in range; four of them are not)
    hb, yb = h.clone(), y.clone()
    hb[at], yb[at] = big, big
    u, got = pdn.pdn_residual_norm(torch.zeros_like(hb), hb, weight=w)
    assert torch.equal(got, hb) and (u[at] == 0).all() and not (u[ok] == 0).all(1).any()
    a, b = pdn.pdn_residual_norm_bwd(du, h, dh=dh, weight=w), pdn.pdn_residual_norm_bwd(du, hb, dh=dh, weight=w)
    for n in ("dy", "dresidual"):
        assert b[n][at].isnan().all() and torch.equal(a[n][ok], b[n][ok]), n
    assert b["dweight"].isnan().all()
    kw = dict(weight=w, post_norm=True, post_weight=w, scale=w)
    u, got = pdn.pdn_residual_norm(yb, h, **kw)
    assert torch.equal(got[at], h[at])   # (the normed y is zeros)
    a, b = pdn.pdn_residual_norm_bwd(du, h, y, dh=dh, **kw), pdn.pdn_residual_norm_bwd(du, h, yb, dh=dh, **kw)
    assert b["dy"][at].isnan().all() and torch.equal(a["dy"][ok], b["dy"][ok])
    assert torch.equal(a["dresidual"], b["dresidual"]) and torch.equal(a["dweight"], b["dweight"])
    assert b["dpost_weight"].isnan().all() and b["dscale"].isnan().all()


@pytest.mark.parametrize("d", [5, 33, 128, 200])
@pytest.mark.parametrize("norm", ["rms", "l2"])
@pytest.mark.parametrize("each", [False, True])
def test_heads_whose_squares_leave_fp32(d, norm, each):
    import torch
    import paper_2604_21100_amd as pdn
    torch.manual_seed(d)
    M, H = 3, 2
    for kind in (torch.float32, torch.bfloat16):
        x, dy, z = (torch.randn(M, H, d, device="cuda").to(kind) for _ in range(3))
        w = torch.rand(H, d, device="cuda") if each else torch.rand(d, device="cuda")
        xb = x.clone()
        xb[1, 1] = 1e19
        kw = dict(norm=norm, weight=w, z=z)
        y = pdn.pdn_head_norm(xb, **kw)
        assert (y[1, 1] == 0).all()
        a, b = pdn.pdn_head_norm_bwd(dy, x, **kw), pdn.pdn_head_norm_bwd(dy, xb, **kw)
        for n in ("dx", "dz"):
            assert b[n][1, 1].isnan().all(), n
            b[n][1, 1] = a[n][1, 1]
            assert torch.equal(a[n], b[n]), n
        assert (b["dweight"][1] if each else b["dweight"]).isnan().all()
        if each:
            assert torch.equal(a["dweight"][0], b["dweight"][0])


@pytest.mark.parametrize("act", ["silu", "sigmoid"])
@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_a_weights_gradient_of_gated_rows_is_fp32s(act, dt):
    """dweight is fp32 for bf16 rows too.  Rows of ones with ones as gradient have a factor of one and a sum of one
    term, so dweight is act(z) as computed.  Relative roundings, in u = 2^-24: the exponential two (a step), its
    correction one; 1 + e, its reciprocal (two where it is the hardware's alone), the product with e and that with z one each: 7 or 8.  (The argument's own
    rounding, up to |z| u, is what the correction puts back.)"""
    import torch
    import paper_2604_21100_amd as pdn
    kind = torch.bfloat16 if dt == "bf16" else torch.float32
    H, d = 512, 128
    z = torch.linspace(-80, 80, H * d, device="cuda").to(kind).view(1, H, d)
    one = torch.ones(1, H, d, device="cuda").to(kind)
    g = pdn.pdn_head_norm_bwd(one, one, weight=torch.ones(H, d, device="cuda"), z=z, act=act, eps=1e-30)
    x = z.double().cpu().numpy()[0]
    s = np.where(x >= 0, 1 / (1 + np.exp(-np.abs(x))), np.exp(-np.abs(x)) / (1 + np.exp(-np.abs(x))))
    want = x * s if act == "silu" else s
    off = np.abs(g["dweight"].double().cpu().numpy() - want)
    assert (off <= 8 * U * np.abs(want)).all(), float((off / np.maximum(np.abs(want), 1e-300)).max() / U)


def test_no_workspace_without_a_vectors_gradient():
    """The parts are the vectors' gradients': a call that wants none needs no workspace."""
    import torch
    import paper_2604_21100_amd as pdn
    torch.manual_seed(1)
    du, h, dh, w = torch.randn(700, 640, device="cuda"), torch.randn(700, 640, device="cuda"), torch.randn(700, 640, device="cuda"), torch.randn(640, device="cuda")
    none = torch.empty(0, dtype=torch.uint8, device="cuda")
    want = pdn.pdn_residual_norm_bwd(du, h, dh=dh, weight=w)
    got = pdn.pdn_residual_norm_bwd(du, h, dh=dh, weight=w, want_vectors=False, workspace=none)
    assert set(got) == {"dy", "dresidual"} and all(torch.equal(got[n], want[n]) for n in got)
    got = pdn.pdn_residual_norm_bwd(du, h, dh=dh, workspace=none)   # (no vectors at all)
    assert set(got) == {"dy", "dresidual"}
    with pytest.raises(pdn.PdnError):
        pdn.pdn_residual_norm_bwd(du, h, dh=dh, weight=w, workspace=none)
