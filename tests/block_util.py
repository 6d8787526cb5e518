"""What the calls around the rule have to return, in 64 bits from their definitions, with
a magnitude for every value: what its terms add up to without cancelling, by which
rounding errors are bounded.

Bounds (u = 2^-24, half a step of fp32): a row's sum of squares is off by at most 40 u
(16 terms in a thread, 6 + 16 over the threads), its factor by 24 u; a gradient through one
norm by 40 + 3 * 24 and a few single roundings, 128 u of its magnitude; one behind two norms by
320 u.  Outputs are rounded once more, by half a step of their own type."""
import numpy as np

U = 2.0 ** -24
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}
ONE, TWO = 128 * U, 320 * U


def dtype(io):
    import torch
    return torch.bfloat16 if io == "bf16" else torch.float32


def seen(x, io):
    """x as the device holds it, in 64 bits."""
    import torch
    return torch.from_numpy(np.asarray(x)).to(dtype(io)).double().numpy()


def close(got, want, mag, io, bound, name=""):
    g = got.double().cpu().numpy()
    assert g.shape == want.shape, (name, g.shape, want.shape)
    room = HALF[io] * np.abs(want) + bound * mag * (1 + HALF[io])
    off = np.abs(g - want)
    assert np.isfinite(g).all(), name
    assert (off <= room).all(), (name, float((off / np.maximum(room, 1e-300)).max()))


def _or1(x):
    return 1.0 if x is None else x


def _factor(x, eps, width):
    return 1 / np.sqrt((x * x).sum(-1, keepdims=True) / width + eps)


def rnorm(y, residual, weight, post, post_weight, scale, alpha, eps):
    """((u, mag), (h, mag))"""
    D = y.shape[-1]
    a = y * _factor(y, eps, D) * _or1(post_weight) if post else y
    b = alpha * _or1(scale) * a
    h = b if residual is None else residual + b
    mh = np.abs(b) + (0 if residual is None else np.abs(residual))
    r = _factor(h, eps, D)
    # (an error of h moves its factor too, by at most as much)
    rel = np.sqrt((mh * mh).sum(-1, keepdims=True) / np.maximum((h * h).sum(-1, keepdims=True), 1e-300))
    return (h * r * _or1(weight), (mh + np.abs(h) * np.minimum(rel, 1e6)) * r * np.abs(_or1(weight))), (h, mh)


def _pull(x, g, mg, eps, width):
    r = _factor(x, eps, width)
    n = x * r
    along = lambda z: (z * n).sum(-1, keepdims=True) / width   # noqa: E731
    return r * (g - n * along(g)), r * (mg + np.abs(n) * (mg * np.abs(n)).sum(-1, keepdims=True) / width)


def rnorm_bwd(du, dh, h, y, weight, post, post_weight, scale, alpha, eps):
    D = h.shape[-1]
    n = h * _factor(h, eps, D)
    t, mt = _pull(h, du * _or1(weight), np.abs(du * _or1(weight)), eps, D)
    if dh is not None:
        t, mt = t + dh, mt + np.abs(dh)
    out = {"dresidual": (t, mt), "dweight": ((du * n).sum(0), np.abs(du * n).sum(0))}
    b, mb = alpha * _or1(scale) * t, np.abs(alpha * _or1(scale)) * mt
    if y is not None:
        m = y * _factor(y, eps, D)
        a = m * _or1(post_weight) if post else y
        out["dscale"] = ((alpha * t * a).sum(0), np.abs(alpha * mt * a).sum(0))
    if post:
        out["dpost_weight"] = ((b * m).sum(0), (mb * np.abs(m)).sum(0))
        b, mb = _pull(y, b * _or1(post_weight), mb * np.abs(_or1(post_weight)), eps, D)
    out["dy"] = (b, mb)
    return out


def act_of(z, act):
    """act(z), its derivative, and the derivative's magnitude"""
    if z is None:
        return 1.0, 0.0, 0.0
    s = np.where(z >= 0, 1 / (1 + np.exp(-np.abs(z))), np.exp(-np.abs(z)) / (1 + np.exp(-np.abs(z))))
    rest = np.where(z >= 0, np.exp(-np.abs(z)) / (1 + np.exp(-np.abs(z))), 1 / (1 + np.exp(-np.abs(z))))
    if act == "silu":
        return z * s, s + z * s * rest, s + np.abs(z) * s * rest
    return s, s * rest, s * rest


def hnorm(x, norm, weight, z, act, eps):
    width = x.shape[-1] if norm == "rms" else 1
    y = x * _factor(x, eps, width) * _or1(weight) * act_of(z, act)[0]
    return y, np.abs(y)


def hnorm_bwd(dy, x, norm, weight, z, act, eps):
    width = x.shape[-1] if norm == "rms" else 1
    a, slope, ms = act_of(z, act)
    w, n = _or1(weight), x * _factor(x, eps, width)
    out = {"dx": _pull(x, dy * w * a, np.abs(dy * w * a), eps, width)}
    if z is not None:
        out["dz"] = dy * w * n * slope, np.abs(dy * w * n) * ms
    if weight is not None:
        dw = dy * n * a
        axes = tuple(range(x.ndim - weight.ndim))
        out["dweight"] = dw.sum(axes), np.abs(dw).sum(axes)
    return out


def changed_logits(l, count, prompt, rep, pres, freq, bias, allowed):
    """A row's logits [V] (float32) after penalties, bias and mask, each step rounded to fp32."""
    f = np.float32
    with np.errstate(all="ignore"):
        l = l.astype(f)
        had = prompt | (count > 0)
        x = np.where(had, np.where(l > 0, (l / f(rep)).astype(f), (l * f(rep)).astype(f)), l)
        y = ((x - (f(freq) * count.astype(f)).astype(f)).astype(f) - f(pres)).astype(f)
        x = np.where(count > 0, y, x)
        x = np.where(bias != 0, (x + bias.astype(f)).astype(f), x)
    return np.where(allowed, x, f(-np.inf))


def probabilities(l, T):
    """(p, bound) of changed logits (float32) [V]; bound: what fp32 may be off, in u of p: the exponent's
    argument has four roundings of its size."""
    V = l.shape[0]
    if np.isnan(l).any():
        return np.full(V, np.nan), np.zeros(V)
    top = l.max() if V else -np.inf
    p = np.zeros(V)
    if not top > -np.inf:
        return p, np.zeros(V)
    if not T > 0:
        p[int(np.argmax(l == top))] = 1.0
        return p, np.zeros(V)
    with np.errstate(all="ignore"):
        arg = np.where(l == top, 0.0, (l.astype(np.float64) - float(top)) / max(float(T), 1e-45))
    arg = np.where(np.isnan(arg), -np.inf, arg)
    e = np.exp(arg)
    size = np.minimum(-arg, 200.0)
    return e / e.sum(), 4 * size + 64 + (e * 4 * size).sum() / e.sum()
