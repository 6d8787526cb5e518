"""pdn_logits with everything on in each of its forms: one launch with one to seven windows a thread, two launches, rows
aligned to an access and not, in place too."""
import numpy as np
import pytest

from test_gpu_logits import Round

pytestmark = pytest.mark.gpu

# rows, vocabulary: windows of one launch (1, 2, 4, 7), then two launches
FORMS = [(3, 1999), (3, 2000), (3, 7999), (3, 16001), (3, 16000), (90, 20001), (90, 32764), (90, 32760), (130, 40003), (130, 57344), (3, 50257),
         (5, 70004), (5, 70003), (5, 70008)]


def batch(rng, rows):
    lens = rng.integers(0, 6, rows)
    ends = np.minimum(np.cumsum(lens), rows)
    lens = np.diff(np.concatenate([[0], ends]))
    return [int(n) for n in lens[lens > 0]] + [rows - int(lens.sum())]


@pytest.mark.parametrize("rows,V", FORMS)
@pytest.mark.parametrize("io", ["f32", "bf16"])
def test_everything_on(rows, V, io):
    rng = np.random.default_rng(rows + V)
    r = Round(rng, batch(rng, rows), V, io, pad=[0, 8, 3][V % 3], greedy=True)
    r.check(rows=range(rows) if rows < 10 else sorted(rng.choice(rows, 10, replace=False)))


@pytest.mark.parametrize("rows,V", FORMS)
@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("probs", [True, False])
def test_in_place(rows, V, io, probs, monkeypatch):
    """The result in the logits' place: the bits of the call that does not, twice the same."""
    import torch
    import paper_2604_21100_amd as pdn
    rng = np.random.default_rng(rows + V)
    r = Round(rng, batch(rng, rows), V, io, greedy=True)
    with monkeypatch.context() as m:
        m.setattr(pdn, "pdn_logits", lambda logits, **kw: (logits, kw))
        l, kw = r.call(probs=probs)
    before = l.clone()
    want = pdn.pdn_logits(l, dtype=l.dtype, **kw)
    assert torch.equal(l.view(torch.int16 if io == "bf16" else torch.int32), before.view(torch.int16 if io == "bf16" else torch.int32))
    for _ in range(2):
        got = l.clone()
        assert pdn.pdn_logits(got, out=got, **kw) is got
        assert torch.equal(got, want)


@pytest.mark.parametrize("rows,V", [(1, 32768), (64, 32000), (79, 16385), (80, 16385), (256, 36001), (257, 36000), (257, 36001), (1535, 36001),
                                    (1536, 36001), (300, 57344)])
@pytest.mark.parametrize("lists", [False, True])
def test_where_one_launch_and_two_meet(rows, V, lists):
    """By rows, tokens and whether lists change the logits: probabilities against 64 bits, with the bound of block_util."""
    import torch
    import paper_2604_21100_amd as pdn
    from block_util import U
    g = torch.Generator(device="cuda").manual_seed(rows + V)
    l = 2 * torch.randn(rows, V, generator=g, device="cuda")
    T = torch.linspace(0.5, 1.5, rows, device="cuda")
    ids = torch.randint(0, V, (rows,), generator=g, device="cuda")
    p = pdn.pdn_logits(l, temperature=T, **(dict(ids=ids.int(), presence=torch.full((rows,), 0.5, device="cuda")) if lists else {}))
    if lists:
        l[torch.arange(rows, device="cuda"), ids] -= 0.5
    arg = (l.double() - l.double().amax(1, keepdim=True)) / T.double()[:, None]
    e = torch.exp(arg)
    want = e / e.sum(1, keepdim=True)
    bound = U * (64 - 4 * arg + (e * -4 * arg).sum(1, keepdim=True) / e.sum(1, keepdim=True)) * want + 2e-38
    assert ((p.double() - want).abs() <= bound).all()


@pytest.mark.parametrize("N", [63, 64, 65, 4095, 4096, 4097, 5000, 270_000])
@pytest.mark.parametrize("rows_before", [0, 3])
def test_a_rows_sequence_among_many(N, rows_before):
    """Sequences of no, one and a few rows, each with a temperature of its own; rows before the first and behind the
    last belong to none."""
    import torch
    import paper_2604_21100_amd as pdn
    from block_util import U
    g = torch.Generator(device="cuda").manual_seed(N)
    lens = torch.randint(0, 4, (N,), generator=g, device="cuda")
    starts = rows_before + torch.cat([torch.zeros(1, dtype=torch.int64, device="cuda"), torch.cumsum(lens, 0)])
    rows, V = int(starts[-1]) + 2, 12
    l = torch.randn(rows, V, generator=g, device="cuda")
    T = 0.3 + torch.rand(N, generator=g, device="cuda")
    out = torch.full((rows, V), 5.0, device="cuda")
    pdn.pdn_logits(l, temperature=T, starts=starts.int(), out=out)
    assert (out[:rows_before] == 5.0).all() and (out[-2:] == 5.0).all()
    own = slice(rows_before, rows - 2)
    arg = (l[own].double() - l[own].double().amax(1, keepdim=True)) / torch.repeat_interleave(T.double(), lens)[:, None]
    e = torch.exp(arg)
    want = e / e.sum(1, keepdim=True)
    assert ((out[own].double() - want).abs() <= U * (64 - 4 * arg + (e * -4 * arg).sum(1, keepdim=True)) * want).all()
