"""Probabilities of logits at values where roundings or ranges could show."""
import numpy as np
import pytest

from block_util import U
from slot_util import i32  # noqa: F401

pytestmark = pytest.mark.gpu
INF = float("inf")


def f32(x):
    import torch
    return torch.tensor(np.asarray(x, np.float32), device="cuda")


@pytest.mark.parametrize("V", [5, 1000, 5000, 20000, 50257, 131072])
@pytest.mark.parametrize("rows", [3, 130])
def test_probabilities_of_unlikely_tokens(V, rows):
    """p is e over a sum that is one (a single token within 40 of the largest, the others add up to less than
    V e^-40): relative roundings, in u = 2^-24, of the exponential two (a step), of what the others add
    V e^-40 / u = V 7e-11, less than one, and of the argument as much as it is large, as it is rounded once; the factor is
    one.  Differences of logits are whole steps of 2^-10 and so exact."""
    import torch
    import paper_2604_21100_amd as pdn
    g = torch.Generator(device="cuda").manual_seed(V + rows)
    T = torch.tensor([0.31, 0.7, 1.0, 1.37, 2.9] * 26, device="cuda")[:rows]
    span = torch.rand(rows, V, generator=g, device="cuda") * 46 + 40.5   # (so e down to 2.7e-38, above the smallest number of 24 bits)
    l = -(span * T[:, None] * 1024).round() / 1024
    top = torch.randint(0, V, (rows, 1), generator=g, device="cuda")
    l.scatter_(1, top, 0.0)
    p = pdn.pdn_logits(l, temperature=T).double()
    arg = -l.double() / T.double()[:, None]
    e = torch.exp(-arg)
    want = e / e.sum(1, keepdim=True)
    off = (p - want).abs() / want
    assert (off <= (arg + 4) * U).all(), (off / (arg + 4)).max().item() / U


@pytest.mark.parametrize("V", [4, 3000, 70000])
def test_the_largest_temperatures(V):
    """Temperatures up to the largest number and infinity, over logits as far apart as they are.  1 / T is held to
    2^-24 down to 1.2e-38 and to 2^-149 below (2e-7 of 1 / 3e38), infinity as 2^-149, which moves a
    logit of -3.4e38 by 5e-7; a token's e so by 1e-6 at most, and its p by twice that."""
    import torch
    import paper_2604_21100_amd as pdn
    T = [1e29, 1e32, 1e38, 3e38, INF]
    for forms in (1, 200):
        temps = T * forms
        l = torch.full((len(temps), V), -INF, device="cuda")
        for r, t in enumerate(temps):
            x = min(t, 1e38)
            l[r, :4] = f32([0.0, -x, -2 * x, -3.4e38])
        got = pdn.pdn_logits(l, temperature=f32(temps)).double()
        e = torch.exp(l.double() / f32(temps).double()[:, None].clamp(max=1e300))
        want = torch.where(l == -INF, 0.0, e / e.sum(1, keepdim=True))
        for r, t in enumerate(temps):
            if t == INF:
                want[r, :4] = 0.25
        assert ((got - want).abs() <= 4e-6 * want).all(), (V, forms, ((got - want).abs() / want.clamp(min=1e-300)).max().item())
