"""From logits to tokens on the GPU: pdn_logits (changed logits equal to the last bit, probabilities
within the roundings of fp32) and pdn_token_counts (whole numbers: equal)."""
import numpy as np
import pytest

from block_util import HALF, U, changed_logits, dtype, probabilities
from slot_util import i32

pytestmark = pytest.mark.gpu
PROMPT = -2 ** 31
INF, NAN = float("inf"), float("nan")


def f32(x):
    import torch
    return None if x is None else torch.tensor(np.asarray(x, np.float32), device="cuda")


class Round:
    """A packed batch of rows with everything that changes logits, on the host."""

    def __init__(self, rng, lens, V, io, *, counts=True, ids=True, bias=True, mask=True, pad=0, slots=None, greedy=False):
        import torch
        N, M = len(lens), int(sum(lens))
        self.V, self.io, self.M, self.N, self.pad = V, io, M, N, pad
        self.starts = np.concatenate([[0], np.cumsum(lens)])
        l = torch.from_numpy((2.5 * rng.standard_normal((M, V))).astype(np.float32)).to(dtype(io))
        self.logits = l.float().numpy()
        pick = lambda lo, hi: rng.uniform(lo, hi, N).astype(np.float32)   # noqa: E731
        self.T, self.rep, self.pres, self.freq = pick(0.3, 2.0), pick(0.7, 1.6), pick(-0.3, 0.6), pick(-0.1, 0.4)
        if greedy:
            self.T[::2] = 0.0
        self.P = N + 2
        self.slots = rng.permutation(self.P)[:N] if slots is None else np.asarray(slots)
        self.table = None
        if counts:
            self.table = (rng.integers(1, 5, (self.P, V)) * (rng.random((self.P, V)) < 0.1)).astype(np.int64)
            self.prompt = rng.random((self.P, V)) < 0.2
        self.ids = rng.integers(-1, min(V, 40) + 1, M) if ids else None
        self.bias = None
        if bias:
            lists = [rng.integers(-1, V + 1, rng.integers(0, 12)) for _ in range(N)]
            ends = np.concatenate([[0], np.cumsum([len(x) for x in lists])])
            flat = np.concatenate(lists) if lists else np.zeros(0, int)
            self.bias = (ends, flat, rng.choice([0.5, -1.25, 3.0, -INF], len(flat)).astype(np.float32))
        self.masks = None
        if mask:
            self.masks = rng.random((M + 1, V)) < 0.3
            self.masks[0] = False   # leaves nothing
            self.mask_rows = rng.integers(-1, M + 2, M)
            self.mask_rows[:min(M, 2)] = [0, -1][:min(M, 2)]

    def call(self, **kw):
        import torch
        import paper_2604_21100_amd as pdn
        wide = torch.full((self.M, self.V + self.pad), NAN, dtype=dtype(self.io), device="cuda")
        wide[:, :self.V] = torch.from_numpy(self.logits).to(dtype(self.io))
        a = dict(temperature=f32(self.T), repetition=f32(self.rep), presence=f32(self.pres), frequency=f32(self.freq), starts=i32(self.starts))
        if self.table is not None:
            t = self.table + np.where(self.prompt, PROMPT, 0)
            a.update(counts=torch.tensor(t, dtype=torch.int32, device="cuda"), slots=i32(self.slots))
        if self.ids is not None:
            a["ids"] = i32(self.ids)
        if self.bias is not None:
            a["bias"] = (i32(self.bias[0]), i32(self.bias[1]), f32(self.bias[2]))
        if self.masks is not None:
            words = -(-self.V // 32)
            bits = np.zeros((len(self.masks), words * 32), np.uint8)
            bits[:, :self.V] = self.masks
            packed = np.packbits(bits, axis=1, bitorder="little").view(np.int32)
            a.update(mask=torch.from_numpy(packed.copy()).cuda(), mask_rows=i32(self.mask_rows))
        a.update(kw)
        return pdn.pdn_logits(wide[:, :self.V], **a)

    def changed(self, row):
        """The row's changed logits, and its temperature; None where it is left out."""
        n = int(np.searchsorted(self.starts, row, side="right")) - 1
        if n < 0 or n >= self.N or (self.table is not None and not 0 <= self.slots[n] < self.P):
            return None, None
        count, prompt = np.zeros(self.V, int), np.zeros(self.V, bool)
        if self.table is not None:
            count, prompt = self.table[self.slots[n]].copy(), self.prompt[self.slots[n]]
        if self.ids is not None:
            for j in self.ids[self.starts[n]:row + 1]:
                if 0 <= j < self.V:
                    count[j] += 1
        bias = np.zeros(self.V, np.float32)
        if self.bias is not None:
            for i in range(self.bias[0][n], self.bias[0][n + 1]):   # (the last entry of a token holds)
                if 0 <= self.bias[1][i] < self.V:
                    bias[self.bias[1][i]] = self.bias[2][i]
        allowed = np.ones(self.V, bool)
        if self.masks is not None and 0 <= self.mask_rows[row] < len(self.masks):
            allowed = self.masks[self.mask_rows[row]]
        return changed_logits(self.logits[row], count, prompt, self.rep[n], self.pres[n], self.freq[n], bias, allowed), self.T[n]

    def check(self, out=None, rows=None, **kw):
        l, p = self.call(probs=False, dtype=dtype("f32"), **kw).cpu().numpy(), self.call(**kw).double().cpu().numpy()
        h = self.call(dtype=dtype("bf16"), **kw).double().cpu().numpy()
        for row in range(self.M) if rows is None else rows:
            want, T = self.changed(row)
            assert np.array_equal(l[row], want, equal_nan=True), row
            wp, bound = probabilities(want, T)
            room = U * bound * wp + 2e-38
            assert np.array_equal(np.isnan(p[row]), np.isnan(wp))
            ok = ~np.isnan(wp)
            assert (np.abs(p[row] - wp) <= room)[ok].all(), (row, np.abs(p[row] - wp).max())
            assert (np.abs(h[row] - wp) <= room * 1.01 + HALF["bf16"] * wp)[ok].all(), row


@pytest.mark.parametrize("V", [1, 7, 8, 33, 2047, 2049, 5000, 50257])
@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("parts", ["all", "counts", "ids", "bias", "mask", "none"])
def test_logits(V, io, parts):
    on = {n: parts in ("all", n) for n in ("counts", "ids", "bias", "mask")}
    r = Round(np.random.default_rng(V), [3, 0, 1, 5, 2], V, io, pad=[0, 3, 128][V % 3], greedy=parts in ("all", "none"), **on)
    r.check()


@pytest.mark.parametrize("V", [131072, 100003])
def test_large_vocabulary(V):
    Round(np.random.default_rng(V), [2, 3], V, "f32").check()
    Round(np.random.default_rng(V), [2, 1], V, "bf16", greedy=True).check()


@pytest.mark.parametrize("N,V", [(1, 3000), (65, 40), (130, 2500), (700, 9)])
def test_many_sequences(N, V):
    """More sequences than a wave has lanes; one row each; the rows shared out without starts."""
    rng = np.random.default_rng(N)
    r = Round(rng, rng.integers(0, 3, N), V, "f32", greedy=True)
    r.check()
    r = Round(rng, [2] * N, V, "bf16", mask=False)
    r.check(starts=None)


def test_a_long_sequence():
    """A sequence of more rows than a workgroup has threads: row t counts all of its tokens up to t."""
    r = Round(np.random.default_rng(5), [700, 3], 64, "f32")
    r.check()


def test_what_is_left_out():
    """Slots outside the pool, rows of no sequence: as they were.  Numbers in `starts` outside the rows are clamped."""
    import torch
    rng = np.random.default_rng(6)
    r = Round(rng, [2, 2, 3], 300, "f32", slots=[1, -1, 99])
    for probs in (True, False):
        out = torch.full((r.M, r.V), 5.0, device="cuda")
        assert r.call(out=out, probs=probs) is out
        assert (out[2:] == 5.0).all() and not (out[:2] == 5.0).any()
    r = Round(rng, [2, 3], 300, "f32", counts=False)
    out = torch.full((r.M, r.V), 5.0, device="cuda")
    starts = r.starts.copy()
    r.call(out=out, starts=i32([1, 3, 4]))
    assert (out[0] == 5.0).all() and (out[4] == 5.0).all() and not (out[1:4] == 5.0).any()
    a = r.call(starts=i32([-7, starts[1], 1000]))
    assert torch.equal(a, r.call())
    out.fill_(5.0)
    r.call(out=out, starts=i32([900, -3, 2]))   # (any numbers: nothing outside the tensors)


def test_no_rows_no_sequences():
    import torch
    import paper_2604_21100_amd as pdn
    e = torch.empty(0, 50, device="cuda")
    assert pdn.pdn_logits(e).shape == (0, 50)
    out = torch.full((2, 50), 5.0, device="cuda")
    pdn.pdn_logits(torch.zeros(2, 50, device="cuda"), starts=i32([0]), out=out)
    assert (out == 5.0).all()


def rows_of(values, **kw):
    import torch
    import paper_2604_21100_amd as pdn
    l = torch.tensor(values, dtype=torch.float32, device="cuda")
    return pdn.pdn_logits(l, **kw).cpu().numpy()


def test_infinities_and_nan():
    assert rows_of([[INF, 1.0, INF, -INF]]).tolist() == [[0.5, 0.0, 0.5, 0.0]]
    assert rows_of([[-INF, -INF]]).tolist() == [[0.0, 0.0]]
    assert rows_of([[-INF, -INF]], temperature=f32([0.0])).tolist() == [[0.0, 0.0]]
    assert rows_of([[1.0, INF, INF]], temperature=f32([0.0])).tolist() == [[0.0, 1.0, 0.0]]
    assert np.isnan(rows_of([[1.0, NAN, 2.0, -INF]])).all()
    assert np.isnan(rows_of([[NAN] * 5000], temperature=f32([0.0]))).all()
    assert np.isnan(rows_of([[0.0] * 3000 + [NAN] + [-1e30] * 3000], temperature=f32([1e-3]))).all()
    assert np.isnan(rows_of([[-INF] * 2048 + [NAN] + [-INF] * 2047 + [1.0]])).all()
    low = np.finfo(np.float32).min
    assert rows_of([[low, low, 0.0]]).tolist() == [[0.0, 0.0, 1.0]]
    assert rows_of([[low, low]]).tolist() == [[0.5, 0.5]]
    # a mask over NaN and infinities
    import torch
    mask = torch.tensor([[0b0100]], dtype=torch.int32, device="cuda")
    assert rows_of([[NAN, INF, 3.0, NAN]], mask=mask).tolist() == [[0.0, 0.0, 1.0, 0.0]]
    assert rows_of([[NAN, INF, 3.0, NAN]], mask=mask, probs=False).tolist() == [[-INF, -INF, 3.0, -INF]]


@pytest.mark.parametrize("T,want", [(0.0, [0, 1, 0, 0]), (-1.0, [0, 1, 0, 0]), (NAN, [0, 1, 0, 0]), (1e-44, [0, 0.5, 0.5, 0]),
                                    (1e-20, [0, 0.5, 0.5, 0]), (INF, [1 / 3, 1 / 3, 1 / 3, 0]), (3e38, [1 / 3, 1 / 3, 1 / 3, 0])])
def test_temperatures(T, want):
    """Zero, below, NaN: the lowest of the largest; the smallest and largest numbers."""
    got = rows_of([[1.0, 2.0, 2.0, -INF]], temperature=f32([T]))
    assert np.allclose(got, [want], rtol=1e-6, atol=0)


def test_lowest_token_of_several():
    """Ties over segments of a long row, in a lane's tokens and across lanes."""
    for at in ([5, 6], [7, 8], [2047, 2048], [100, 60000], [40001, 40003, 65000]):
        l = np.zeros((1, 66000), np.float32)
        l[0, at] = 3.0
        got = rows_of(l.tolist(), temperature=f32([0.0]))
        assert got[0, at[0]] == 1.0 and got.sum() == 1.0


def test_in_place():
    import torch
    import paper_2604_21100_amd as pdn
    torch.manual_seed(1)
    for dt in (torch.float32, torch.bfloat16):
        l = torch.randn(5, 9001, device="cuda").to(dt)
        ids = i32(range(5))
        want = pdn.pdn_logits(l, ids=ids, dtype=dt, repetition=f32([1.5] * 5))
        got = pdn.pdn_logits(l.clone(), ids=ids, repetition=f32([1.5] * 5), dtype=dt)
        assert torch.equal(got, want)
        assert pdn.pdn_logits(l, ids=ids, repetition=f32([1.5] * 5), out=l) is l and torch.equal(l, want)


def test_verification_reads_it():
    """A row that the mask leaves nothing of: the verification says -1."""
    import torch
    import paper_2604_21100_amd as pdn
    p = pdn.pdn_logits(torch.randn(2, 100, device="cuda"), mask=torch.zeros(2, 4, dtype=torch.int32, device="cuda"), mask_rows=i32([1, -1]))
    acc, tok = pdn.pdn_draft_verify(p, i32([3, 4]), f32([0.5, 0.5]), f32([0.5, 0.5]))
    assert acc.tolist() == [1, 1] and tok[0] == -1 and tok[1] >= 0


@pytest.mark.parametrize("rows,V", [(95, 16385), (96, 16384), (96, 16385), (97, 32769), (96, 57344), (96, 57345), (3, 16384), (3, 16385),
                                    (79, 16385), (80, 16385), (80, 32768), (127, 32769), (128, 32769),
                                    (128, 57344), (128, 57345), (5, 2048), (5, 2049), (5, 8192), (5, 8193), (4, 32768), (300, 70000)])
def test_where_the_forms_meet(rows, V):
    """One launch or two go by rows and tokens: every token's probability against 64 bits, a greedy row among them."""
    import torch
    import paper_2604_21100_amd as pdn
    g = torch.Generator(device="cuda").manual_seed(V)
    l = 2 * torch.randn(rows, V, generator=g, device="cuda")
    l[rows // 2, 5:9] = 50.0
    T = torch.linspace(0.5, 1.5, rows, device="cuda")
    T[rows // 2] = 0.0
    p = pdn.pdn_logits(l, temperature=T)
    assert p[rows // 2].nonzero().tolist() == [[5]] and p[rows // 2, 5] == 1.0
    live = torch.arange(rows, device="cuda") != rows // 2
    arg = (l.double() - l.double().amax(1, keepdim=True)) / T.double()[:, None]
    e = torch.exp(arg)
    want = e / e.sum(1, keepdim=True)
    bound = U * (64 - 4 * arg + (e * -4 * arg).sum(1, keepdim=True) / e.sum(1, keepdim=True)) * want + 2e-38
    assert ((p.double() - want).abs() <= bound)[live].all()


def test_offsets_past_32_bits():
    """The last rows of tensors of more than 2^31 elements, and of such a table: the bits of a small call."""
    import torch
    import paper_2604_21100_amd as pdn
    R, V, n = 17000, 131072, 2
    g = torch.Generator(device="cuda").manual_seed(3)
    l = torch.zeros(R, V, dtype=torch.bfloat16, device="cuda")
    l[-n:] = torch.randn(n, V, generator=g, device="cuda")
    table = torch.zeros(R, V, dtype=torch.int32, device="cuda")
    pdn.pdn_token_counts(i32([3, V - 1, 3]), table, starts=i32([0, 3]), slots=i32([R - 1]))
    assert table[R - 1].nonzero()[:, 0].tolist() == [3, V - 1] and table[R - 1, 3] == 2 and not table[:R - 1].any()
    pdn.pdn_token_counts(i32([7]), table, starts=i32([0, 1]), slots=i32([R - 1]), slots_out=i32([R - 2]), prompt=True)
    assert table[R - 2].nonzero()[:, 0].tolist() == [3, 7, V - 1] and not table[:R - 2].any()
    kw = dict(repetition=f32([1.5] * R), frequency=f32([0.3] * R), dtype=torch.bfloat16)
    big = pdn.pdn_logits(l, counts=table, **kw)
    kw = dict(repetition=f32([1.5] * n), frequency=f32([0.3] * n), dtype=torch.bfloat16)
    small = pdn.pdn_logits(l[-n:], counts=table, slots=i32([R - 2, R - 1]), **kw)
    # (sums of as many segments, but not of the same: the same to a step of bf16)
    assert ((big[-n:].float() - small.float()).abs() <= 2 ** -7 * small.float()).all()
    assert (big[0].float() - 1 / V).abs().max() <= 2 ** -8 / V
    assert torch.equal(pdn.pdn_logits(l, counts=table, probs=False, repetition=f32([1.5] * R))[-n:],
                       pdn.pdn_logits(l[-n:], counts=table, slots=i32([R - 2, R - 1]), probs=False, repetition=f32([1.5] * n)))


# ---------------------------------------------------------------- counts
def ref_counts(table, ids, starts, slots, slots_out, fresh, accepted, prompt):
    new = table.copy()
    V = table.shape[1]
    for n in range(len(starts) - 1):
        a = int(slots[n])
        b = a if slots_out is None else int(slots_out[n])
        if not (0 <= a < len(table) and 0 <= b < len(table)):
            continue
        row = (new if slots_out is None else table)[a].copy()
        if fresh is not None and fresh[n]:
            row[:] = 0
        toks = ids[starts[n]:starts[n + 1]]
        if accepted is not None:
            toks = toks[:max(accepted[n], 0)]
        for j in toks:
            if 0 <= j < V:
                row[j] = row[j] | PROMPT if prompt else row[j] + 1
        new[b] = row
    return new


@pytest.mark.parametrize("V", [1, 50, 2048, 2049, 50257])
@pytest.mark.parametrize("prompt", [False, True])
@pytest.mark.parametrize("form", ["add", "fresh", "fork", "both"])
def test_counts(V, prompt, form):
    import torch
    import paper_2604_21100_amd as pdn
    rng = np.random.default_rng(V + prompt)
    P, lens = 14, [3, 0, 400, 1, 20, 7]
    table = (rng.integers(0, 4, (P, V)) + np.where(rng.random((P, V)) < 0.3, PROMPT, 0)).astype(np.int64)
    starts = np.concatenate([[0], np.cumsum(lens)])
    ids = rng.integers(-1, min(V, 30) + 1, starts[-1])
    perm = rng.permutation(P)
    slots = perm[:6].copy()
    slots[4] = 99 if form != "add" else -1
    out = perm[6:12].copy() if form in ("fork", "both") else None
    if out is not None:
        out[0] = slots[0]    # stays where it is
        out[3] = -5
    fresh = rng.integers(0, 2, 6) if form in ("fresh", "both") else None
    for accepted in (None, np.array([2, 5, 1000, -1, 3, 0])):
        want = ref_counts(table, ids, starts, slots, out, fresh, accepted, prompt)
        t = torch.tensor(table, dtype=torch.int32, device="cuda")
        got = pdn.pdn_token_counts(i32(ids), t, starts=i32(starts), slots=i32(slots), slots_out=i32(out), fresh=i32(fresh),
                                   accepted=i32(accepted), prompt=prompt)
        assert got is t
        assert np.array_equal(t.cpu().numpy().astype(np.int64), want)


def test_counts_defaults():
    """Without starts and slots a token each; with accepted the rows shared out."""
    import torch
    import paper_2604_21100_amd as pdn
    t = torch.zeros(3, 9, dtype=torch.int32, device="cuda")
    pdn.pdn_token_counts(i32([4, 4, 8]), t)
    assert t.nonzero().tolist() == [[0, 4], [1, 4], [2, 8]]
    pdn.pdn_token_counts(i32([1, 2, 3, 1, 2, 3]), t, accepted=i32([3, 1]))
    assert t[0].tolist() == [0, 1, 1, 1, 1, 0, 0, 0, 0] and t[1].tolist() == [0, 1, 0, 0, 1, 0, 0, 0, 0]
    pdn.pdn_token_counts(i32([5, 5]), t, slots=i32([2, 2]))   # two sequences that add to one slot
    assert t[2].tolist() == [0, 0, 0, 0, 0, 2, 0, 0, 1]
    pdn.pdn_token_counts(i32([]), t, starts=i32([0, 0]), fresh=i32([1]))
    assert t[0].sum() == 0 and t[1].sum() == 2


# ---------------------------------------------------------------- together
@pytest.mark.parametrize("graph", [False, True])
def test_rounds_of_a_server(graph):
    """Logits -> pdn_logits -> pdn_draft_verify -> pdn_token_counts over rounds, eager and as a captured graph that is
    replayed with new inputs and eager calls between: every table row and every choice is the host's."""
    import torch
    import paper_2604_21100_amd as pdn
    rng = np.random.default_rng(11)
    N, K, V, P = 3, 4, 3000, 5
    M = N * K
    table = np.zeros((P, V), np.int64)
    prompts = [rng.integers(0, 60, 30) for _ in range(N)]
    slots = np.array([4, 0, 2])
    counts = torch.zeros(P, V, dtype=torch.int32, device="cuda")
    flat = np.concatenate(prompts)
    pdn.pdn_token_counts(i32(flat), counts, starts=i32([0, 30, 60, 90]), slots=i32(slots), fresh=i32([1, 1, 1]), prompt=True)
    table = ref_counts(table, flat, [0, 30, 60, 90], slots, None, [1, 1, 1], None, True)
    logits = torch.empty(M, V, device="cuda")
    ids, u, r = torch.empty(M, dtype=torch.int32, device="cuda"), torch.empty(M, device="cuda"), torch.empty(N, device="cuda")
    kw = dict(temperature=f32([0.0, 0.8, 1.3]), repetition=f32([1.3, 1.0, 1.1]), presence=f32([0.1, 0.4, 0.0]), frequency=f32([0.0, 0.2, 0.3]))
    sl, starts = i32(slots), i32([0, K, 2 * K, 3 * K])
    p, acc, tok = torch.empty(M, V, device="cuda"), torch.empty(N, dtype=torch.int32, device="cuda"), torch.empty(N, dtype=torch.int32, device="cuda")
    ws = torch.empty(pdn.pdn_logits_workspace_size(M, V), dtype=torch.uint8, device="cuda")
    wv = torch.empty(pdn.pdn_draft_verify_workspace_size(N, V), dtype=torch.uint8, device="cuda")

    def run():
        pdn.pdn_logits(logits, counts=counts, slots=sl, ids=ids, starts=starts, out=p, workspace=ws, **kw)
        pdn.pdn_draft_verify(p, ids, u, r, starts=starts, accepted=acc, token=tok, workspace=wv)
        pdn.pdn_token_counts(ids, counts, starts=starts, slots=sl, accepted=acc)

    if graph:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            run()
    fed = np.zeros(N, int) + 7
    for _ in range(5):
        l = rng.standard_normal((M, V)).astype(np.float32) * 2
        l[:, :60] += 3.0   # (tokens come again)
        drafts = rng.integers(0, 60, (N, K))
        drafts[:, 0] = fed
        for n in range(N):   # likely drafts: what the row says itself
            for t in range(1, K):
                drafts[n, t] = int(l[n * K + t - 1].argmax())
        ru, rr = rng.random(M).astype(np.float32), rng.random(N).astype(np.float32)
        logits.copy_(torch.from_numpy(l)); ids.copy_(torch.from_numpy(drafts.reshape(-1).astype(np.int32)))   # noqa: E702
        u.copy_(torch.from_numpy(ru)); r.copy_(torch.from_numpy(rr))   # noqa: E702
        before = table.copy()
        if graph:
            g.replay()
        else:
            run()
        got_p, got_acc, got_tok = p.double().cpu().numpy(), acc.cpu().numpy(), tok.cpu().numpy()
        for n in range(N):
            row = before[slots[n]]
            count = row & 0x7fffffff
            for t in range(K):
                count[drafts[n, t]] += 1
                want = changed_logits(l[n * K + t], count, row < 0, kw["repetition"][n].item(), kw["presence"][n].item(),
                                      kw["frequency"][n].item(), np.zeros(V, np.float32), np.ones(V, bool))
                wp, bound = probabilities(want, kw["temperature"][n].item())
                assert (np.abs(got_p[n * K + t] - wp) <= U * bound * wp + 2e-38).all()
            held = 0   # (a draft without probabilities of its own: u < p)
            while held + 1 < K and ru[n * K + held] < got_p[n * K + held][drafts[n, held + 1]]:
                held += 1
            assert got_acc[n] == held + 1
        table = ref_counts(table, drafts.reshape(-1), [0, K, 2 * K, 3 * K], slots, None, None, got_acc, False)
        assert np.array_equal(counts.cpu().numpy().astype(np.int64), table)
        fed = got_tok
        eager = pdn.pdn_logits(logits, temperature=kw["temperature"], starts=starts)   # (an eager call between replays)
        assert eager.shape == (M, V)


def test_other_streams_and_two_graphs():
    """Calls in flight on two streams with workspaces of their own; two captured graphs replayed in turn."""
    import torch
    import paper_2604_21100_amd as pdn
    torch.manual_seed(3)
    a, b = torch.randn(6, 70000, device="cuda"), torch.randn(9, 50001, device="cuda").bfloat16()
    want = [pdn.pdn_logits(a), pdn.pdn_logits(b)]
    side = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for _ in range(3):
        got = [pdn.pdn_logits(x, stream=s) for x, s in zip((a, b), side)]
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(want, got))
    graphs = []
    for x, w in zip((a, b), want):
        out, ws = torch.empty_like(w), torch.empty(pdn.pdn_logits_workspace_size(*x.shape), dtype=torch.uint8, device="cuda")
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            pdn.pdn_logits(x, out=out, workspace=ws)
        graphs.append((g, out, ws))
    for _ in range(3):
        for (g, out, _), w in zip(graphs, want):
            out.fill_(-1.0)
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, w)
