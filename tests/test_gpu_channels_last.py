"""Tensors [N][C][H][W] whose memory is [N][H][W][C], as PyTorch's channels_last keeps them, go through the training
operators as they lie: the same bits as for [N][H][W][C] itself."""
import pytest

pytestmark = pytest.mark.gpu


def test_operators_take_them_as_they_lie():
    import torch
    import paper_2004_11077_amd as wn
    N, C, H, W, V = 2, 24, 5, 7, 11
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda")
    rows = N * H * W
    nhwc, dy = r(N, H, W, C), r(N, H, W, C)
    w, target, dloss = r(V, C), torch.randint(0, V, (N, H, W), generator=g, device="cuda"), r(N, H, W)
    nd, ld, od = wn.NormDesc(rows, C), wn.LossDesc(rows, C, V), wn.OrthogonaliseDesc(1, C, 9 * V)
    room = lambda n: torch.empty(n, dtype=torch.uint8, device="cuda")
    last = lambda t: t.permute(0, 3, 1, 2)       # what channels_last is
    out = []
    for see in (lambda t: t, last):
        y, mean, rstd = see(torch.empty_like(nhwc)), *r(2, N, H, W)
        wn.wino_layer_norm(nd, see(nhwc), None, None, y, mean, rstd)
        dx, dgamma = see(torch.empty_like(nhwc)), r(C)
        wn.wino_layer_norm_backward(nd, see(dy), see(nhwc), None, mean, rstd, dx, dgamma, None,
                                    room(wn.wino_layer_norm_backward_workspace_bytes(nd)))
        loss, lse = r(2, N, H, W)
        ws = room(max(wn.wino_linear_cross_entropy_workspace_bytes(ld), wn.wino_linear_cross_entropy_backward_workspace_bytes(ld)))
        wn.wino_linear_cross_entropy(ld, see(nhwc), w, None, target, loss, lse, ws)
        dh, dw = see(torch.empty_like(nhwc)), torch.empty_like(w)
        wn.wino_linear_cross_entropy_backward(ld, see(nhwc), w, None, target, lse, dloss, dh, dw, None, ws)
        out.append([t.permute(0, 2, 3, 1) if see is last and t.dim() == 4 else t for t in (y, mean, rstd, dx, dgamma, loss, lse, dh, dw)])
    assert all(torch.equal(a, b) for a, b in zip(*out))
    # filters: the columns stand in another order, and so do the result's, up to the sums' roundings
    grad = r(C, V, 3, 3)
    o, p = torch.empty_like(grad), torch.empty_like(grad, memory_format=torch.channels_last)
    ws = room(wn.wino_orthogonalise_workspace_bytes(od))
    wn.wino_orthogonalise(od, grad, o, ws)
    wn.wino_orthogonalise(od, grad.to(memory_format=torch.channels_last), p, ws)
    # five steps, each of which makes an error up to four times as large, of sums of 99 products in fp32, factor 10.3
    assert (o - p).norm() <= 4 ** 5 * 10.3 * 2 * (8 + 2 * 99 ** 0.5) * 2.0 ** -24 * o.norm()
