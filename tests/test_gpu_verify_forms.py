"""pdn_draft_verify where its forms meet: one launch or two go by the sequences and the
vocabulary."""
import numpy as np
import pytest

from slot_util import dev, i32
from test_gpu_draft import probs, ref_verify

pytestmark = pytest.mark.gpu


def drafts(rng, N, V, dtype, given, live):
    """N sequences of which the first, the last and `live - 2` between have rows."""
    import torch
    lens = np.zeros(N, int)
    at = sorted({0, N - 1} | set(rng.permutation(N)[:max(live - 2, 0)].tolist()))
    lens[at] = rng.integers(1, 5, len(at))
    starts = np.concatenate([[0], np.cumsum(lens)])
    M = int(starts[-1])
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    p, P = probs(rng, M, V, dt)
    q, Q = probs(rng, M, V, dt) if given else (None, None)
    ids = rng.integers(0, V, M)
    u, r = (0.5 * rng.random(M)).astype(np.float32), rng.random(N).astype(np.float32)
    if given:
        for t in range(1, M, 2):   # some drafts from the target itself
            q[t], Q[t] = p[t - 1], P[t - 1]
    want = ref_verify(P, Q, ids, u.astype(np.float64), r.astype(np.float64), starts)
    return (p, i32(ids), dev(u), dev(r)), dict(q=q, starts=i32(starts)), want


@pytest.mark.parametrize("N,V", [(1, 24576), (1, 24768), (1, 24769), (64, 32000), (64, 32768), (64, 32769), (64, 36864),
                                 (64, 36865), (214, 65536), (214, 65537), (500, 65535), (3, 40000)])
@pytest.mark.parametrize("dtype,given", [("f32", True), ("bf16", False)])
def test_where_the_forms_meet(N, V, dtype, given):
    import paper_2604_21100_amd as pdn
    args, kw, want = drafts(np.random.default_rng(N + V), N, V, dtype, given, 5)
    acc, tok = pdn.pdn_draft_verify(*args, **kw)
    assert (acc.cpu().tolist(), tok.cpu().tolist()) == want
