"""Workspace sizes of the norms' backward calls from Python, on the host."""
import ctypes

import pytest

pdn = pytest.importorskip("paper_2604_21100_amd", reason="libpdn.so not built")


@pytest.mark.parametrize("rows,D", [(0, 5), (1, 1), (999, 1001), (16384, 2048), (70, 16384)])
def test_residual_norm(rows, D):
    n = ctypes.c_size_t()
    for io in (pdn.PDN_F32, pdn.PDN_BF16):   # (the same for every kind of call)
        for post in (0, 1):
            p = pdn.Rnorm(rows=rows, D=D, io=io, stream=pdn.PDN_F32, post_norm=post, alpha=0.5, eps=1e-6)
            assert pdn._lib.pdn_residual_norm_bwd_workspace_size(ctypes.byref(p), ctypes.byref(n)) == pdn.PDN_OK
            assert pdn.pdn_residual_norm_bwd_workspace_size(rows, D) == n.value
    assert (n.value > 0) == (rows > 0)


@pytest.mark.parametrize("tokens,H,d", [(0, 2, 8), (1, 1, 1), (300, 0, 16), (16384, 16, 128), (2, 5000, 16)])
@pytest.mark.parametrize("each", [False, True])
def test_head_norm(tokens, H, d, each):
    n = ctypes.c_size_t()
    for act in pdn.ACTS.values():
        p = pdn.Hnorm(tokens=tokens, H=H, d=d, io=pdn.PDN_BF16, norm=1, act=act, head_weight=int(each), eps=1e-6, x_stride=H * d + 8)
        assert pdn._lib.pdn_head_norm_bwd_workspace_size(ctypes.byref(p), ctypes.byref(n)) == pdn.PDN_OK
        assert pdn.pdn_head_norm_bwd_workspace_size(tokens, H, d, each) == n.value
    assert (n.value > 0) == (tokens * H > 0)


def test_refusals():
    for call in (lambda: pdn.pdn_residual_norm_bwd_workspace_size(-1, 5), lambda: pdn.pdn_residual_norm_bwd_workspace_size(1, 0),
                 lambda: pdn.pdn_residual_norm_bwd_workspace_size(1, 16385), lambda: pdn.pdn_head_norm_bwd_workspace_size(-1, 1, 1),
                 lambda: pdn.pdn_head_norm_bwd_workspace_size(1, 1, 513)):
        with pytest.raises(pdn.PdnError):
            call()


@pytest.mark.gpu
@pytest.mark.parametrize("rows,D", [(999, 1001), (3000, 640), (700, 24), (600, 9000)])
def test_a_workspace_of_that_size_is_enough_and_less_is_not(rows, D):
    import torch
    torch.manual_seed(D)
    du, h, y, w = torch.randn(rows, D, device="cuda"), torch.randn(rows, D, device="cuda"), torch.randn(rows, D, device="cuda"), torch.randn(D, device="cuda")
    kw = dict(weight=w, post_norm=True, post_weight=w, scale=w)
    n = pdn.pdn_residual_norm_bwd_workspace_size(rows, D)
    room = torch.full((n + 256,), 7, dtype=torch.uint8, device="cuda")
    got, want = pdn.pdn_residual_norm_bwd(du, h, y, workspace=room[:n], **kw), pdn.pdn_residual_norm_bwd(du, h, y, **kw)
    assert all(torch.equal(got[k], want[k]) for k in want) and (room[n:] == 7).all()
    with pytest.raises(pdn.PdnError):
        pdn.pdn_residual_norm_bwd(du, h, y, workspace=room[:n - 1], **kw)
    H, d = (5, D // 5) if D % 5 == 0 else (1, 24)
    for each in (False, True):
        x, dy = (t[:, :H * d].reshape(-1, H, d) if d <= 512 else t.view(-1, H * 10, d // 10) for t in (h, du))
        M, K, e = x.shape
        wx = torch.randn(K, e, device="cuda") if each else torch.randn(e, device="cuda")
        n = pdn.pdn_head_norm_bwd_workspace_size(M, K, e, each)
        room = torch.full((n + 256,), 7, dtype=torch.uint8, device="cuda")
        got, want = pdn.pdn_head_norm_bwd(dy, x, weight=wx, workspace=room[:n]), pdn.pdn_head_norm_bwd(dy, x, weight=wx)
        assert all(torch.equal(got[k], want[k]) for k in want) and (room[n:] == 7).all()
        with pytest.raises(pdn.PdnError):
            pdn.pdn_head_norm_bwd(dy, x, weight=wx, workspace=room[:n - 1])
