"""The compiled part of the binding on the host: rows of tokens that it must not take for
dense ones.  (Host tensors are refused too, after everything that is said of shapes and
strides.)"""
import pytest

pdn = pytest.importorskip("paper_2604_21100_amd", reason="libpdn.so not built")
torch = pytest.importorskip("torch")


def wrong_rows(M, n, d):
    """[M, n, d] tensors whose tokens' rows share memory."""
    one = torch.zeros(1, n, d)
    yield one.expand(M, n, d)                                               # a row for all tokens
    yield torch.zeros(M * n * d).as_strided((M, n, d), (n * d - 8, d, 1))   # a row reaches into the next
    yield torch.zeros(M * n * d).as_strided((M, n, d), (8, d, 1))


@pytest.mark.parametrize("draft", [False, True])
@pytest.mark.parametrize("name", ["q", "k", "v"])
@pytest.mark.parametrize("Hk", [1, 2])
def test_rows_that_share_memory_are_refused(name, Hk, draft):
    M, H, d = 6, 2, 64
    shapes = dict(q=Hk, k=Hk, v=H)
    for wrong in wrong_rows(M, shapes[name], d):
        a = {n: torch.zeros(M, h, d) for n, h in shapes.items()}
        a[name] = wrong
        S, beta = torch.zeros(M, H, d, d), torch.zeros(M, H)
        with pytest.raises(ValueError, match=f"row of {name} .* overlap"):
            if draft:
                pdn.pdn_slot_draft(a["q"], a["k"], a["v"], beta, S, torch.zeros(M, 1, H, 2 * d + 4),
                                   torch.zeros(M, H, dtype=torch.int32), precond="identity")
            else:
                pdn.pdn_slot_fwd(a["q"], a["k"], a["v"], beta, S, precond="identity")


def test_rows_of_their_own_pass_that_check():
    """Slices of one projection; one token, whatever its stride says; no token."""
    H, d = 2, 64
    for M, q in ((6, torch.zeros(6, 3 * H * d)[:, :H * d].view(6, H, d)), (1, torch.zeros(1, H, d).expand(1, H, d)),
                 (1, torch.zeros(H * d).as_strided((1, H, d), (0, d, 1))), (0, torch.zeros(1, H, d).expand(0, H, d))):
        rows = torch.zeros(M, H, d)
        with pytest.raises(ValueError, match="S is on cpu"):   # (all that is wrong with them)
            pdn.pdn_slot_fwd(q, rows, rows, torch.zeros(M, H), torch.zeros(8, H, d, d), precond="identity")
