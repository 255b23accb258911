"""The training operators at the ends of their ranges: one row, feature, class or channel and the most of them.
Tolerances: those derived in the operators' own tests."""
import numpy as np
import pytest

from oracle import training as tr
from test_gpu_cross_entropy import check, run
from test_gpu_layer_norm import U
from test_gpu_orthogonalise import compare, gradients, room

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("type", ["f32", "bf16"])
@pytest.mark.parametrize("T,D,V", [(1 << 21, 1, 2), ((1 << 21) - 1, 5, 3), (70001, 1, 1), (70001, 3, 65), (1, 1, 1 << 22), (3, 2, (1 << 22) + 1),
                                   (200, 1, 1 << 18), (1, 1 << 20, 70), (3, (1 << 20) - 1, 5), (193, 1 << 17, 66)])
def test_cross_entropy(T, D, V, type):
    check(run(T, D, V, type, seed=V), type)


@pytest.mark.parametrize("y_type", ["f32", "i8"])
@pytest.mark.parametrize("rows,channels", [(1, 1 << 24), (2, (1 << 24) - 3), (1 << 23, 1), ((1 << 22) + 1, 3), (1 << 21, 16)])
def test_layer_norm(rows, channels, y_type):
    import torch
    import paper_2004_11077_amd as wn
    g = torch.Generator(device="cuda")
    g.manual_seed(channels)
    x, dy = torch.randn(2, rows, channels, generator=g, device="cuda")
    gamma, beta = torch.randn(2, channels, generator=g, device="cuda")
    codes = y_type == "i8"
    desc = wn.NormDesc(rows, channels, y_type=wn.TYPE_I8 if codes else wn.TYPE_F32, s_y=0.03)
    y = torch.empty(rows, channels, device="cuda", dtype=torch.int8 if codes else torch.float32)
    mean, rstd = torch.empty(2, rows, device="cuda")
    wn.wino_layer_norm(desc, x, gamma, beta, y, mean, rstd)
    dx, dgamma, dbeta = torch.empty_like(x), *torch.empty(2, channels, device="cuda")
    ws = torch.empty(wn.wino_layer_norm_backward_workspace_bytes(desc), dtype=torch.uint8, device="cuda")
    wn.wino_layer_norm_backward(desc, dy, x, gamma, mean, rstd, dx, dgamma, dbeta, ws)
    d = lambda t: t.double()
    xd = d(x)
    mu = xd.mean(1, keepdim=True)
    s = 1 / ((xd - mu).square().mean(1, keepdim=True) + float(np.float32(1e-5))).sqrt()
    ref = (xd - mu) * s * gamma + beta
    n = 64 + channels / 1024
    if codes:
        # the order of the 64-bit sums decides values within some 2^-40 of a border
        q = ref / float(np.float32(0.03))
        apart = (q - q.floor() - 0.5).abs() > 2.0 ** -40
        assert torch.equal(d(y)[apart], q.round().clamp(-127, 127)[apart]) and apart.double().mean() > 0.999
    else:
        off = U * (n + 1) * xd.abs().mean(1, keepdim=True)
        plain = (ref - beta).abs()
        # one channel: (x - mean) is zero and s is what eps leaves, 316
        tol = gamma.abs() * s * off + (n + 8) * U * plain + 2 * U * (ref.abs() + beta.abs()) + plain * (off * s) ** 2 / 2
        assert ((d(y) - ref).abs() <= tol).all()
    xh = (xd - d(mean)[:, None]) * d(rstd)[:, None]
    gr = d(dy) * gamma
    m = lambda a: a.mean(1, keepdim=True)
    rdx = d(rstd)[:, None] * (gr - m(gr) - xh * m(gr * xh))
    xa, ga = xh.abs(), gr.abs()
    tol = d(rstd)[:, None] * U * (4 * ga + (n + 4) * m(ga) + (n + 12) * (xa + 1) * m(ga * (xa + 1))) + 4 * U * rdx.abs()
    assert ((d(dx) - rdx).abs() <= tol).all()
    k = rows / 512 + 72
    assert ((d(dgamma) - (d(dy) * xh).sum(0)).abs() <= k * U * (d(dy).abs() * xa).sum(0)).all()
    assert ((d(dbeta) - d(dy).sum(0)).abs() <= k * U * d(dy).abs().sum(0)).all()


@pytest.mark.parametrize("batch,rows,cols", [(65535, 1, 1), (65535, 3, 2), (4097, 17, 65), (1, 1, 1 << 20), (1, 1 << 20, 2), (2, 100001, 33), (7, 64, 74000)])
def test_updates(batch, rows, cols):
    import torch
    import paper_2004_11077_amd as wn
    some = np.unique(np.linspace(0, batch - 1, 16).astype(int))
    g = torch.randn(batch, rows, cols, device="cuda") * 1e-3
    g[torch.from_numpy(some).cuda()] = torch.from_numpy(gradients(len(some), rows, cols, 5)).float().cuda()
    o = torch.full_like(g, float("nan"))
    desc = wn.OrthogonaliseDesc(batch, rows, cols)
    wn.wino_orthogonalise(desc, g, o, room(wn, desc))
    assert torch.isfinite(o).all()
    compare(o.double().cpu().numpy()[some], g.double().cpu().numpy()[some], "f32")
