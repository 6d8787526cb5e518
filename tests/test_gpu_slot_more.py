"""The state-pool calls where other tests leave a gap: verifications in flight on two
streams with workspaces of their own, heads in halves over sequences of many chunks and
of none."""
import numpy as np
import pytest

from slot_util import batch, i32, pool
from test_gpu_slots import check, run, want
from test_gpu_verify_forms import drafts

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("V", [9000, 50257])
def test_two_streams_at_once(V):
    """Calls in flight on two streams, one after the other on each, with what they allocate
    their own: the workspace that a call's first launch leaves its second must not be
    another's meanwhile, whichever stream is current."""
    import torch
    import paper_2604_21100_amd as pdn
    rng = np.random.default_rng(V)
    sets = [drafts(rng, 6, V, "f32", True, 6) for _ in range(4)]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    got = []
    for turn in range(8):   # (named, and as the current one)
        args, kw, want = sets[turn % 4]
        s = streams[turn % 2]
        if turn < 4:
            got.append((pdn.pdn_draft_verify(*args, stream=s, **kw), want))
        else:
            with torch.cuda.stream(s):
                got.append((pdn.pdn_draft_verify(*args, **kw), want))
        junk = torch.full((1 << 14,), float("nan"), device="cuda")   # (the current stream's, as freed workspaces would be)
        del junk
    torch.cuda.synchronize()
    for (acc, tok), want in got:
        assert (acc.cpu().tolist(), tok.cpu().tolist()) == want


@pytest.mark.parametrize("io,gate,precond", [("bf16", "scalar", "identity"), ("bf16", "none", "external"),
                                              ("bf16", "channel", "identity"), ("f32", "scalar", "external")])
@pytest.mark.parametrize("N", [32, 33])
def test_halves_of_uneven_sequences(io, gate, precond, N):
    """128 heads (two workgroups each) and 132: empty sequences, one of four chunks, forks of
    a slot, a new sequence, a padded one."""
    rng = np.random.default_rng(N)
    H, d = 4, 128
    lens = [int(x) for x in rng.integers(0, 40, N)]
    lens[0], lens[3], lens[4], lens[N - 1] = 0, 100, 9, 0
    b = batch(rng, sum(lens), H, H, d, d, io, gate, precond)
    S, A = pool(rng, N + 3, H, d, d, precond)
    src = list(range(N))
    dst = list(src)
    src[5], dst[5] = 2, N          # 2 is read by 2 and 5, and written by 5 elsewhere
    dst[2] = N + 1
    src[6] = -1
    fresh = [int(n in (3, 7, N - 1)) for n in range(N)]
    o, S1, A1, starts = want(b, S, A, lens, gate, precond, src, dst, fresh)
    got = run(b, S, A, io, gate, precond, starts=i32(starts), slots=i32(src), slots_out=i32(dst), fresh=i32(fresh), max_tokens=100)
    check(got, (o, S1, A1), io, 100)
    assert np.array_equal(got[1][N + 2], S[N + 2]) and np.array_equal(got[1][2], S[2])
