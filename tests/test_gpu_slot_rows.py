"""Rows of tokens on the device: what the binding refuses of them, before any launch, and
the strides that it takes."""
import numpy as np
import pytest

from slot_util import KW, batch, dev, dev_batch, host, i32, pool
from test_gpu_slots import check, run, want

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T", [1, 6, 40])
@pytest.mark.parametrize("io", ["bf16", "f32"])
def test_a_row_for_all_tokens(T, io):
    """Expanded over the tokens a row is refused; laid out, or as the only one, it is taken."""
    import paper_2604_21100_amd as pdn
    rng = np.random.default_rng(T)
    N, H, d = 2, 2, 64
    b = batch(rng, N * T, H, 1, d, d, io, "none", "identity")
    for n in "qkv":
        b[n][:] = b[n][:1]
    S, _ = pool(rng, N, H, d, d, "identity")
    pos, _ = dev_batch(b, io, "identity")
    kw = dict(gate="none", precond="identity", starts=i32([0, T, 2 * T]), max_tokens=T, **KW)
    for i in range(3):
        bad = list(pos)
        bad[i] = pos[i][:1].expand(pos[i].shape)
        Sd = dev(S)
        with pytest.raises(ValueError, match="overlap"):
            pdn.pdn_slot_fwd(*bad, Sd, **kw)
        assert np.array_equal(host(Sd), S)
        bad[i] = bad[i].contiguous()
        o = pdn.pdn_slot_fwd(*bad, Sd, **kw)
        ro, rS, _, _ = want(b, S, None, [T, T], "none", "identity")
        check((host(o), host(Sd), None), (ro, rS, None), io, T)
    one = [x[:1].expand(1, *x.shape[1:]) for x in pos]
    Sd = dev(S[:1])
    o = pdn.pdn_slot_fwd(*one, Sd, gate="none", precond="identity", **KW)
    ro, rS, _, _ = want({n: None if x is None else x[:1] for n, x in b.items()}, S[:1], None, [1], "none", "identity")
    check((host(o), host(Sd), None), (ro, rS, None), io, 1)


@pytest.mark.parametrize("gate", ["scalar", "channel"])
def test_no_limit_on_a_sequence(gate):
    """max_tokens past any length, or not given: nothing is cut."""
    rng = np.random.default_rng(3)
    lens, H, d = [5, 0, 70, 1], 2, 128
    b = batch(rng, sum(lens), H, H, d, d, "bf16", gate, "squash")
    S, A = pool(rng, 4, H, d, d, "squash")
    o, S1, A1, starts = want(b, S, A, lens, gate, "squash")
    for most in (None, 2 ** 40, 2 ** 63 - 1):
        check(run(b, S, A, "bf16", gate, "squash", starts=i32(starts), max_tokens=most), (o, S1, A1), "bf16", 70)
