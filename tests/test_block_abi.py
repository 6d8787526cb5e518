"""The calls around the rule on the host: what they refuse, before any HIP call (fake addresses, never
dereferenced; every call here fails validation or has nothing to do), and the definitions that their GPU tests
compare with, against differences."""
import ctypes

import numpy as np
import pytest

import block_util as bu

pdn = pytest.importorskip("paper_2604_21100_amd", reason="libpdn.so not built")

A = 1 << 32   # fake addresses this far apart do not overlap
BIG = 1 << 30


def rnorm(**kw):
    v = dict(rows=8, D=100, io=pdn.PDN_BF16, stream=pdn.PDN_F32, post_norm=1, alpha=1.0, eps=1e-6)
    v.update(kw)
    return pdn.Rnorm(*[v[n] for n, _ in pdn.Rnorm._fields_])


def hnorm(**kw):
    v = dict(tokens=8, H=4, d=64, io=pdn.PDN_BF16, norm=0, act=1, head_weight=0, eps=1e-6, x_stride=0, z_stride=0, y_stride=0, dy_stride=0,
             dx_stride=0, dz_stride=0)
    v.update(kw)
    return pdn.Hnorm(*[v[n] for n, _ in pdn.Hnorm._fields_])


def call_rnorm(p=None, y=A, residual=2 * A, weight=3 * A, post_weight=4 * A, scale=5 * A, u=6 * A, h=7 * A):
    return pdn._lib.pdn_residual_norm(ctypes.byref(p or rnorm()), y, residual, weight, post_weight, scale, u, h, None)


def call_rnorm_bwd(p=None, du=A, dh=2 * A, h=3 * A, y=4 * A, weight=5 * A, post_weight=6 * A, scale=7 * A, dy=8 * A, dresidual=9 * A,
                   dweight=10 * A, dpost_weight=11 * A, dscale=12 * A, ws=13 * A, ws_bytes=BIG):
    return pdn._lib.pdn_residual_norm_bwd(ctypes.byref(p or rnorm()), du, dh, h, y, weight, post_weight, scale, dy, dresidual, dweight,
                                          dpost_weight, dscale, ws, ws_bytes, None)


def call_hnorm(p=None, x=A, z=2 * A, weight=3 * A, y=4 * A):
    return pdn._lib.pdn_head_norm(ctypes.byref(p or hnorm()), x, z, weight, y, None)


def call_hnorm_bwd(p=None, dy=A, x=2 * A, z=3 * A, weight=4 * A, dx=5 * A, dz=6 * A, dweight=7 * A, ws=8 * A, ws_bytes=BIG):
    return pdn._lib.pdn_head_norm_bwd(ctypes.byref(p or hnorm()), dy, x, z, weight, dx, dz, dweight, ws, ws_bytes, None)


NULL, SHAPE, DTYPE, UNSUP, ALIGN, ALIAS, WS, VALUE = (getattr(pdn, "PDN_ERR_" + n) for n in (
    "NULL", "SHAPE", "DTYPE", "UNSUPPORTED", "ALIGN", "ALIAS", "WORKSPACE", "VALUE"))


def test_rnorm_refusals():
    bad = [(rnorm(rows=-1), SHAPE), (rnorm(D=0), SHAPE), (rnorm(D=16385), UNSUP), (rnorm(rows=1 << 47), SHAPE), (rnorm(io=2), DTYPE),
           (rnorm(stream=-1), DTYPE), (rnorm(eps=0.0), VALUE), (rnorm(eps=float("nan")), VALUE), (rnorm(eps=float("inf")), VALUE),
           (rnorm(alpha=float("inf")), VALUE)]
    for p, status in bad:
        assert call_rnorm(p=p) == call_rnorm_bwd(p=p) == status
        n = ctypes.c_size_t()
        assert pdn._lib.pdn_residual_norm_bwd_workspace_size(ctypes.byref(p), ctypes.byref(n)) == status
    assert pdn._lib.pdn_residual_norm(None, A, None, None, None, None, 2 * A, None, None) == NULL
    for kw, status in [(dict(y=None), NULL), (dict(u=None), NULL), (dict(p=rnorm(post_norm=0)), VALUE), (dict(y=A + 1), ALIGN),
                       (dict(residual=2 * A + 2), ALIGN), (dict(weight=3 * A + 2), ALIGN), (dict(h=7 * A + 2), ALIGN), (dict(u=A), ALIAS),
                       (dict(h=A + 64), ALIAS), (dict(u=2 * A), ALIAS), (dict(h=2 * A + 4), ALIAS), (dict(u=7 * A), ALIAS), (dict(u=3 * A), ALIAS),
                       (dict(h=5 * A), ALIAS), (dict(u=2 * A, h=2 * A), ALIAS)]:
        assert call_rnorm(**kw) == status, kw
    assert call_rnorm(p=rnorm(rows=0), y=None, u=None) == pdn.PDN_OK
    for kw, status in [(dict(du=None), NULL), (dict(h=None), NULL), (dict(dy=None), NULL), (dict(y=None), NULL),
                       (dict(p=rnorm(post_norm=0), post_weight=None, dpost_weight=None, y=None), NULL), (dict(weight=None), VALUE),
                       (dict(post_weight=None), VALUE), (dict(scale=None), VALUE), (dict(p=rnorm(post_norm=0)), VALUE), (dict(du=A + 1), ALIGN),
                       (dict(dh=2 * A + 2), ALIGN), (dict(dweight=10 * A + 1), ALIGN), (dict(dy=A), ALIAS), (dict(dresidual=3 * A), ALIAS),
                       (dict(dresidual=2 * A + 4), ALIAS), (dict(dweight=5 * A), ALIAS), (dict(dscale=10 * A), ALIAS), (dict(ws=A - BIG + 64), ALIAS),
                       (dict(ws=None), WS), (dict(ws_bytes=100), WS), (dict(ws=13 * A + 16), WS)]:
        assert call_rnorm_bwd(**kw) == status, kw
    assert pdn._lib.pdn_residual_norm_bwd_workspace_size(ctypes.byref(rnorm()), None) == NULL


def test_hnorm_refusals():
    bad = [(hnorm(tokens=-1), SHAPE), (hnorm(H=-1), SHAPE), (hnorm(d=0), SHAPE), (hnorm(d=513), UNSUP), (hnorm(H=1 << 24), SHAPE), (hnorm(H=1 << 21), SHAPE),
           (hnorm(tokens=1 << 45), SHAPE), (hnorm(io=5), DTYPE), (hnorm(norm=2), VALUE), (hnorm(act=3), VALUE), (hnorm(eps=-1.0), VALUE)]
    for p, status in bad:
        assert call_hnorm(p=p) == call_hnorm_bwd(p=p) == status
        n = ctypes.c_size_t()
        assert pdn._lib.pdn_head_norm_bwd_workspace_size(ctypes.byref(p), ctypes.byref(n)) == status
    assert pdn._lib.pdn_head_norm(None, A, None, None, 2 * A, None) == NULL
    for kw, status in [(dict(x=None), NULL), (dict(z=None), NULL), (dict(y=None), NULL), (dict(p=hnorm(act=0)), VALUE), (dict(x=A + 1), ALIGN),
                       (dict(weight=3 * A + 2), ALIGN), (dict(y=2 * A), ALIAS), (dict(y=A + 2), ALIAS), (dict(y=3 * A), ALIAS),
                       (dict(p=hnorm(x_stride=255)), SHAPE), (dict(p=hnorm(z_stride=-256)), SHAPE), (dict(p=hnorm(y_stride=1 << 50)), SHAPE),
                       (dict(p=hnorm(x_stride=512), y=A), ALIAS),                           # in place, but of another stride
                       (dict(p=hnorm(x_stride=512, y_stride=512), y=A + 256), ALIAS),       # columns that overlap
                       (dict(p=hnorm(x_stride=512, y_stride=520), y=A + 512), ALIAS)]:      # strides that differ
        assert call_hnorm(**kw) == status, kw
    for kw, status in [(dict(dy=None), NULL), (dict(dx=None), NULL), (dict(dz=None), NULL), (dict(p=hnorm(act=0)), VALUE), (dict(weight=None), VALUE),
                       (dict(dx=2 * A), ALIAS), (dict(dz=5 * A), ALIAS), (dict(dz=A), ALIAS), (dict(dweight=4 * A), ALIAS), (dict(dz=6 * A + 1), ALIGN),
                       (dict(p=hnorm(dx_stride=512, dz_stride=512), dz=5 * A + 400), ALIAS), (dict(p=hnorm(dz_stride=8)), SHAPE), (dict(ws=None), WS),
                       (dict(ws_bytes=64), WS), (dict(ws=8 * A + 8), WS), (dict(ws=7 * A), ALIAS)]:
        assert call_hnorm_bwd(**kw) == status, kw
    none = hnorm(tokens=0)
    assert call_hnorm(p=none) == pdn.PDN_OK and call_hnorm_bwd(p=none, weight=None, dweight=None, ws=None, ws_bytes=0) == pdn.PDN_OK
    n = ctypes.c_size_t(9)
    assert pdn._lib.pdn_head_norm_bwd_workspace_size(ctypes.byref(hnorm(H=0)), ctypes.byref(n)) == pdn.PDN_OK and n.value == 0
    assert call_hnorm_bwd(p=hnorm(H=0, head_weight=1), dy=None, x=None, z=None, dx=None, dz=None) == pdn.PDN_OK


def logits_args(**kw):
    v = dict(rows=6, V=100, N=3, dtype=pdn.PDN_F32, out_dtype=pdn.PDN_F32, probs=1, stride=0, logits=A, starts=2 * A, temperature=3 * A,
             repetition=4 * A, presence=5 * A, frequency=6 * A, counts=7 * A, slots=5, slot=8 * A, ids=9 * A, bias_starts=10 * A, bias_ids=11 * A,
             bias_values=12 * A, biases=7, mask=13 * A, masks=4, mask_rows=14 * A)
    v.update(kw)
    return pdn.LogitsArgs(*[v[n] for n, _ in pdn.LogitsArgs._fields_])


def call_logits(out=15 * A, ws=16 * A, ws_bytes=BIG, **kw):
    return pdn._lib.pdn_logits(ctypes.byref(logits_args(**kw)), out, ws, ws_bytes, None)


def test_logits_refusals():
    for kw, status in [(dict(rows=-1), SHAPE), (dict(V=-1), SHAPE), (dict(V=0), SHAPE), (dict(N=-1), SHAPE), (dict(rows=1 << 31), SHAPE),
                       (dict(V=1 << 31), SHAPE), (dict(rows=1 << 24), SHAPE), (dict(slots=-1), SHAPE), (dict(biases=-1), SHAPE), (dict(masks=-1), SHAPE),
                       (dict(starts=None, N=4), SHAPE), (dict(starts=None, N=0), SHAPE), (dict(slot=None, slots=2), SHAPE),
                       (dict(mask_rows=None), SHAPE), (dict(stride=99), SHAPE), (dict(dtype=2), DTYPE), (dict(out_dtype=2), DTYPE),
                       (dict(logits=None), NULL), (dict(out=None), NULL), (dict(bias_ids=None), NULL), (dict(bias_values=None), NULL),
                       (dict(bias_starts=None), NULL), (dict(counts=None), VALUE), (dict(mask=None), VALUE), (dict(logits=A + 2), ALIGN),
                       (dict(out=15 * A + 1, out_dtype=pdn.PDN_BF16), ALIGN), (dict(temperature=3 * A + 2), ALIGN), (dict(out=7 * A), ALIAS),
                       (dict(out=A + 400), ALIAS), (dict(out=A, out_dtype=pdn.PDN_BF16), ALIAS), (dict(out=A, stride=128), ALIAS),
                       (dict(out=9 * A), ALIAS), (dict(out=13 * A + 16), ALIAS), (dict(ws=15 * A), ALIAS), (dict(ws=None), WS), (dict(ws_bytes=80), WS),
                       (dict(ws=16 * A + 64), WS)]:
        assert call_logits(**kw) == status, (kw, status)
    assert pdn._lib.pdn_logits(None, A, None, 0, None) == NULL
    assert call_logits(rows=0) == call_logits(N=0) == pdn.PDN_OK
    assert call_logits(rows=0, logits=None, out=None, ws=None, ws_bytes=0) == pdn.PDN_OK
    assert pdn._lib.pdn_logits_workspace_size(4, 5, None) == NULL
    with pytest.raises(pdn.PdnError):
        pdn.pdn_logits_workspace_size(-1, 5)
    assert pdn.pdn_logits_workspace_size(0, 0) == 0


def call_counts(N=3, rows=9, V=50, slots=5, prompt=0, ids=A, starts=2 * A, slot=3 * A, slot_out=4 * A, fresh=5 * A, accepted=6 * A, counts=7 * A):
    return pdn._lib.pdn_token_counts(N, rows, V, slots, prompt, ids, starts, slot, slot_out, fresh, accepted, counts, None)


def test_counts_refusals():
    for kw, status in [(dict(N=-1), SHAPE), (dict(rows=-1), SHAPE), (dict(V=-1), SHAPE), (dict(slots=-1), SHAPE), (dict(N=1 << 24), SHAPE),
                       (dict(N=1 << 20, V=1 << 17), SHAPE), (dict(rows=10, starts=None), SHAPE), (dict(slot=None, slots=2), SHAPE),
                       (dict(V=1 << 31), SHAPE), (dict(ids=None), NULL), (dict(counts=None), NULL), (dict(ids=A + 2), ALIGN),
                       (dict(counts=7 * A + 1), ALIGN), (dict(counts=A), ALIAS), (dict(accepted=7 * A + 8), ALIAS)]:
        assert call_counts(**kw) == status, (kw, status)
    assert call_counts(N=0) == call_counts(slots=0, V=0) == pdn.PDN_OK


def test_host_tensors_are_refused():
    """The compiled part of the binding, without a GPU: tensors on the host, of wrong kinds, shapes and spacings."""
    torch = pytest.importorskip("torch")
    z = torch.zeros
    y, i = z(4, 64), z(4, dtype=torch.int32)
    on_host = "is on cpu"
    for call, err, text in [
            (lambda: pdn.pdn_residual_norm(y), ValueError, on_host),
            (lambda: pdn.pdn_residual_norm(y.half()), TypeError, "float32 or bfloat16"),
            (lambda: pdn.pdn_residual_norm(y, z(4, 63)), ValueError, "residual must be"),
            (lambda: pdn.pdn_residual_norm(y, y.double()), TypeError, "float32 or bfloat16"),
            (lambda: pdn.pdn_residual_norm(y, y, h_dtype=torch.bfloat16), TypeError, "h_dtype"),
            (lambda: pdn.pdn_residual_norm(y, h_dtype=torch.int32), TypeError, "float32 or bfloat16"),
            (lambda: pdn.pdn_residual_norm(y.T), ValueError, "contiguous"),
            (lambda: pdn.pdn_residual_norm(y, weight=z(63)), ValueError, "weight must be"),
            (lambda: pdn.pdn_residual_norm(y, weight=z(64).bfloat16()), TypeError, "weight must be"),
            (lambda: pdn.pdn_residual_norm_bwd(y, y), ValueError, on_host),
            (lambda: pdn.pdn_residual_norm_bwd(y, z(5, 64)), ValueError, "h must be"),
            (lambda: pdn.pdn_residual_norm_bwd(y, y, y.bfloat16()), TypeError, "y must be"),
            (lambda: pdn.pdn_head_norm(z(4, 2, 64)), ValueError, on_host),
            (lambda: pdn.pdn_head_norm(z(4)), ValueError, "H, d"),
            (lambda: pdn.pdn_head_norm(z(4, 2, 128)[..., ::2]), ValueError, "dense"),
            (lambda: pdn.pdn_head_norm(z(4, 64, 2).transpose(1, 2)), ValueError, "dense"),
            (lambda: pdn.pdn_head_norm(z(1, 2, 64).expand(4, 2, 64)), ValueError, "overlap"),
            (lambda: pdn.pdn_head_norm(z(3, 4, 2, 64).transpose(0, 1)), ValueError, "evenly"),
            (lambda: pdn.pdn_head_norm(z(3, 5, 2, 64)[:, :4]), ValueError, "evenly"),
            (lambda: pdn.pdn_head_norm(z(4, 2, 64), weight=z(2, 63)), ValueError, "weight must be"),
            (lambda: pdn.pdn_head_norm(z(4, 2, 64), z=z(4, 2, 63)), ValueError, "z must be"),
            (lambda: pdn.pdn_head_norm_bwd(z(4, 2, 64), z(4, 2, 64)), ValueError, on_host),
            (lambda: pdn.pdn_head_norm_bwd(z(4, 2, 64), z(4, 2, 64), weight=z(64), outputs=dict(dweight=z(2, 64))), ValueError, "dweight must be"),
            (lambda: pdn.pdn_logits(z(4, 9)), ValueError, on_host),
            (lambda: pdn.pdn_logits(z(4)), ValueError, "rows, V"),
            (lambda: pdn.pdn_logits(z(9, 4).T), ValueError, "dense"),
            (lambda: pdn.pdn_logits(z(1, 9).expand(4, 9)), ValueError, "overlap"),
            (lambda: pdn.pdn_logits(z(4, 9), ids=z(4)), TypeError, "ids must be"),
            (lambda: pdn.pdn_logits(z(4, 9), temperature=z(2), presence=z(4)), ValueError, "presence must be"),
            (lambda: pdn.pdn_logits(z(4, 9), counts=z(4, 8, dtype=torch.int32)), ValueError, "counts must be"),
            (lambda: pdn.pdn_logits(z(4, 9), mask=z(4, 2, dtype=torch.int32)), ValueError, "mask must be"),
            (lambda: pdn.pdn_logits(z(4, 9), bias=(i, i)), ValueError, "bias must be"),
            (lambda: pdn.pdn_logits(z(4, 9), bias=(i, i, z(4))), ValueError, "bias starts must be"),
            (lambda: pdn.pdn_logits(z(4, 9), starts=z(0, dtype=torch.int32)), ValueError, "one entry more"),
            (lambda: pdn.pdn_token_counts(i, z(4, 9, dtype=torch.int32)), ValueError, on_host),
            (lambda: pdn.pdn_token_counts(i, z(4, 9)), TypeError, "counts must be"),
            (lambda: pdn.pdn_token_counts(i, z(9, dtype=torch.int32)), ValueError, "slots, V"),
            (lambda: pdn.pdn_token_counts(i, z(4, 9, dtype=torch.int32), accepted=i[:3], slots=i), ValueError, "accepted must be")]:
        with pytest.raises(err, match=text):
            call()
    for name, call in (("norm", lambda: pdn.pdn_head_norm(z(1, 1, 2), norm="max")), ("act", lambda: pdn.pdn_head_norm(z(1, 1, 2), act="relu"))):
        with pytest.raises(KeyError):
            call()


def differences(f, x, v, step=1e-5):
    return (f(x + step * v) - f(x - step * v)) / (2 * step)


@pytest.mark.parametrize("post,scale", [(False, False), (True, True), (False, True), (True, False)])
def test_residual_norm_gradients_against_differences(post, scale):
    rng = np.random.default_rng(1)
    f = rng.standard_normal
    p = dict(y=f((3, 6)), residual=f((3, 6)), weight=f(6), post_weight=f(6) if post else None, scale=f(6) if scale else None)
    du, dh = f((3, 6)), f((3, 6))

    def value(**kw):
        a = dict(p, **kw)
        (u, _), (h, _) = bu.rnorm(a["y"], a["residual"], a["weight"], post, a["post_weight"], a["scale"], 0.7, 0.3)
        return (du * u).sum() + (dh * h).sum()

    h = bu.rnorm(p["y"], p["residual"], p["weight"], post, p["post_weight"], p["scale"], 0.7, 0.3)[1][0]
    g = bu.rnorm_bwd(du, dh, h, p["y"], p["weight"], post, p["post_weight"], p["scale"], 0.7, 0.3)
    for n, x in p.items():
        if x is None:
            continue
        v = f(x.shape)
        d = differences(lambda t: value(**{n: t}), x, v)   # noqa: B023
        # (central differences: step^2 of the third derivative, 1e-10 of values of order 10)
        assert abs(d - (g["d" + n][0] * v).sum()) <= 1e-7 * max(1, abs(d)), n


@pytest.mark.parametrize("norm,act,weight", [("rms", "silu", (5,)), ("l2", "none", None), ("rms", "sigmoid", (2, 5)), ("l2", "silu", (2, 5))])
def test_head_norm_gradients_against_differences(norm, act, weight):
    rng = np.random.default_rng(2)
    f = rng.standard_normal
    p = dict(x=f((3, 2, 5)), z=None if act == "none" else f((3, 2, 5)), weight=None if weight is None else f(weight))
    dy = f((3, 2, 5))
    value = lambda **kw: (dy * bu.hnorm(dict(p, **kw)["x"], norm, dict(p, **kw)["weight"], dict(p, **kw)["z"], act, 0.2)[0]).sum()   # noqa: E731
    g = bu.hnorm_bwd(dy, p["x"], norm, p["weight"], p["z"], act, 0.2)
    for n, x in p.items():
        if x is None:
            continue
        v = f(x.shape)
        d = differences(lambda t: value(**{n: t}), x, v)   # noqa: B023
        assert abs(d - (g["d" + n][0] * v).sum()) <= 1e-7 * max(1, abs(d)), n
