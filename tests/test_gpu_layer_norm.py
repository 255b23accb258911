"""Layer norm and its backward pass: the library against the formulas in 64 bits.

Tolerances, element by element, with u = 2^-24.  A sum over a row is taken by lanes of at most
16 values each (1/1024 of a longer row) and a tree of at most ten steps and sixteen waves: with n = 64 + C / 1024 it is
off by at most n u times the sum of magnitudes.  So the mean is off by n u mean|x|, the variance
(sums of squares, the mean's own error entering squared) by (n + 4) u of itself, 1 / sqrt by half of
that, and y by |gamma| s n u mean|x| + (n + 8) u |gamma xh| + 2 u |y|.  The backward pass takes mean
and rstd as given, so xh has 3 u; its two sums have (n + 8) u of their magnitudes, and a column
sum over R rows, taken in 512 parts, at most (R / 512 + 64) u of its magnitudes more.  A bf16 result is rounded
once more, by half a step, 2^-8 of itself.  Codes are computed in 64 bits and equal the formula's.
"""
import numpy as np
import pytest

from oracle import training as tr

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
TYPES = {"f32": 0, "bf16": 1, "i8": 2}


def torch_type(name):
    import torch
    return {"f32": torch.float32, "bf16": torch.bfloat16, "i8": torch.int8}[name]


def padded(rows, channels, stride, dtype, offset=0, fill=None):
    """A device tensor [rows][channels] with `stride` elements between rows, `offset` from an
    aligned address, and the whole allocation behind it."""
    import torch
    whole = torch.full((offset + rows * stride + 64,), 7 if fill is None else fill, device="cuda").to(dtype)
    return whole[offset:offset + rows * stride].view(rows, stride)[:, :channels], whole


def case(rows, channels, x_type, stride, offset, seed, scale=1.0):
    import torch
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((rows, channels)) * scale * (0.5 + rng.random(channels)) + scale * rng.standard_normal(channels)
    t, _ = padded(rows, channels, stride, torch_type(x_type), offset)
    t.copy_(torch.from_numpy(x))
    gamma = (1 + 0.2 * rng.standard_normal(channels)).astype(np.float32)
    beta = (0.2 * rng.standard_normal(channels)).astype(np.float32)
    return t, gamma, beta


SHAPES = [  # rows, channels, extra stride, offset in elements
    (1, 1, 0, 0), (3, 2, 0, 0), (64, 16, 0, 0), (5, 16, 16, 0), (257, 64, 0, 0), (33, 80, 0, 0), (7, 100, 4, 0),
    (19, 144, 0, 1), (100, 256, 0, 0), (13, 255, 0, 0), (9, 512, 0, 3), (6, 1000, 24, 0), (4, 1026, 0, 0), (5, 2048, 0, 0),
    (3, 2049, 0, 0), (3, 4096, 0, 0), (2, 8192, 0, 0), (2, 8200, 8, 0), (3, 16384, 0, 0), (2, 20001, 0, 0)]


@pytest.mark.parametrize("types", [("f32", "f32"), ("f32", "bf16"), ("f32", "i8"), ("bf16", "f32"), ("bf16", "bf16"), ("bf16", "i8")])
@pytest.mark.parametrize("rows,channels,extra,offset", SHAPES)
def test_forward(rows, channels, extra, offset, types):
    import torch
    import paper_2004_11077_amd as wn
    xt, yt = types
    stride = channels + extra
    x, gamma, beta = case(rows, channels, xt, stride, offset, seed=rows + channels)
    s_y, eps = 3.0 / 127, 1e-5
    desc = wn.NormDesc(rows, channels, x_type=TYPES[xt], y_type=TYPES[yt], eps=eps, s_y=s_y, x_stride=stride, y_stride=stride)
    y, whole = padded(rows, channels, stride, torch_type(yt), offset)
    mean, rstd = torch.empty(2, rows, device="cuda")
    wn.wino_layer_norm(desc, x, torch.from_numpy(gamma).cuda(), torch.from_numpy(beta).cuda(), y, mean, rstd)
    torch.cuda.synchronize()
    xd = x.double().cpu().numpy()
    ref, rmean, rrstd = tr.layer_norm(xd, gamma.astype(np.float64), beta.astype(np.float64), np.float64(np.float32(eps)))
    n = 64 + channels / 1024
    off = U * (n + 1) * np.abs(xd).mean(1)
    assert (np.abs(mean.cpu().numpy() - rmean) <= off + U * np.abs(rmean)).all()
    spread = off ** 2 * rrstd ** 2 / 2
    assert (np.abs(rstd.cpu().numpy() / rrstd - 1) <= (n / 2 + 6) * U + spread).all()
    got = y.double().cpu().numpy()
    if yt == "i8":
        assert np.array_equal(got, tr.codes(ref, s_y).astype(np.float64))
    else:
        plain = np.abs(ref - beta)
        tol = np.abs(gamma) * (rrstd * off)[:, None] + (n + 8) * U * plain + plain * spread[:, None] + 2 * U * (np.abs(ref) + np.abs(beta))
        tol += 2.0 ** -8 * np.abs(ref) if yt == "bf16" else 0
        assert (np.abs(got - ref) <= tol).all()
    # nothing beside the rows is written
    mark = torch.full_like(whole, 7)
    mark[offset:offset + rows * stride].view(rows, stride)[:, :channels] = y
    assert torch.equal(whole, mark)


def test_forward_without_optional_tensors():
    import torch
    import paper_2004_11077_amd as wn
    x = torch.randn(37, 96, device="cuda")
    y, z = torch.empty_like(x), torch.empty_like(x)
    desc = wn.NormDesc(37, 96)
    wn.wino_layer_norm(desc, x, None, None, y)
    wn.wino_layer_norm(desc, x, torch.ones(96, device="cuda"), torch.zeros(96, device="cuda"), z)
    assert torch.equal(y, z)


def test_rows_of_one_value_and_rows_with_nan():
    import torch
    import paper_2004_11077_amd as wn
    x = torch.randn(6, 70, device="cuda")
    x[1] = 3.25
    x[3, 17] = float("nan")
    x[4, 2] = float("inf")
    beta = torch.randn(70, device="cuda")
    y = torch.empty_like(x)
    wn.wino_layer_norm(wn.NormDesc(6, 70), x, None, beta, y)
    assert torch.equal(y[1], beta)                       # no spread: (x - mean) is zero
    assert torch.isnan(y[3]).all() and torch.isnan(y[4]).any()
    assert torch.isfinite(y[[0, 1, 2, 5]]).all()
    q = torch.empty(6, 70, dtype=torch.int8, device="cuda")
    wn.wino_layer_norm(wn.NormDesc(6, 70, y_type=wn.TYPE_I8, s_y=0.02), x, None, beta, q)
    assert not q[3].any()                                # the code of a NaN is zero


def test_large_mean_and_small_spread():
    """The variance is no difference of large sums: 1000 +- 1 in fp32 keeps (n + 8) u 1000 of y."""
    import torch
    import paper_2004_11077_amd as wn
    rng = np.random.default_rng(5)
    xn = (1000 + rng.standard_normal((50, 320))).astype(np.float32)
    y = torch.empty(50, 320, device="cuda")
    wn.wino_layer_norm(wn.NormDesc(50, 320), torch.from_numpy(xn).cuda(), None, None, y)
    ref, _, rstd = tr.layer_norm(xn, 1.0, 0.0, np.float64(np.float32(1e-5)))
    tol = 72 * U * (1000 * rstd[:, None] + np.abs(ref) + 1)
    assert (np.abs(y.cpu().numpy() - ref) <= tol).all()


@pytest.mark.parametrize("types", [("f32", "f32"), ("f32", "bf16"), ("bf16", "f32"), ("bf16", "bf16")])
@pytest.mark.parametrize("rows,channels,extra,offset", SHAPES + [(4099, 64, 0, 0), (2050, 24, 0, 0)])
def test_backward(rows, channels, extra, offset, types):
    import torch
    import paper_2004_11077_amd as wn
    xt, gt = types
    stride = channels + extra
    x, gamma, _ = case(rows, channels, xt, stride, offset, seed=3 * rows + channels)
    rng = np.random.default_rng(channels)
    dy, _ = padded(rows, channels, stride, torch_type(gt), offset)
    dy.copy_(torch.from_numpy(rng.standard_normal((rows, channels))))
    xd, dyd = x.double().cpu().numpy(), dy.double().cpu().numpy()
    _, mean, rstd = tr.layer_norm(xd, 1.0, 0.0, 1e-5)
    mean, rstd = mean.astype(np.float32), rstd.astype(np.float32)
    desc = wn.NormDesc(rows, channels, x_type=TYPES[xt], g_type=TYPES[gt], x_stride=stride, dy_stride=stride, dx_stride=stride)
    dx, whole = padded(rows, channels, stride, torch_type(gt), offset)
    dgamma, dbeta = torch.full((2, channels), float("nan"), device="cuda")
    ws = torch.full((wn.wino_layer_norm_backward_workspace_bytes(desc),), 255, dtype=torch.uint8, device="cuda")
    t = lambda a: torch.from_numpy(a).cuda()
    args = (dy, x, t(gamma), t(mean), t(rstd))
    wn.wino_layer_norm_backward(desc, *args, dx, dgamma, dbeta, ws)
    torch.cuda.synchronize()
    rdx, rdg, rdb = tr.layer_norm_backward(dyd, xd, gamma.astype(np.float64), mean, rstd)
    n = 64 + channels / 1024
    xh, g = np.abs((xd - mean[:, None]) * rstd[:, None]), np.abs(dyd * gamma)
    m = lambda a: a.mean(1, keepdims=True)
    tol = rstd[:, None] * U * (4 * g + (n + 4) * m(g) + (n + 12) * (xh + 1) * m(g * (xh + 1))) + 4 * U * np.abs(rdx)
    tol += 2.0 ** -8 * np.abs(rdx) if gt == "bf16" else 0
    assert (np.abs(dx.double().cpu().numpy() - rdx) <= tol).all()
    k = rows / 512 + 64 + 8
    assert (np.abs(dgamma.cpu().numpy() - rdg) <= k * U * (np.abs(dyd) * xh).sum(0) + U * np.abs(rdg)).all()
    assert (np.abs(dbeta.cpu().numpy() - rdb) <= k * U * np.abs(dyd).sum(0) + U * np.abs(rdb)).all()
    mark = torch.full_like(whole, 7)
    mark[offset:offset + rows * stride].view(rows, stride)[:, :channels] = dx
    assert torch.equal(whole, mark)
    # each output alone, and the whole again: the same bits
    only = torch.empty_like(dgamma)
    wn.wino_layer_norm_backward(desc, *args, None, only, None, ws)
    assert torch.equal(only, dgamma)
    wn.wino_layer_norm_backward(desc, *args, None, None, only, ws)
    assert torch.equal(only, dbeta)
    again, _ = padded(rows, channels, stride, torch_type(gt), offset)
    wn.wino_layer_norm_backward(desc, *args, again, None, None, None)
    assert torch.equal(again, dx)


def test_no_rows():
    import torch
    import paper_2004_11077_amd as wn
    for channels in (48, 20001):
        desc = wn.NormDesc(0, channels)
        wn.wino_layer_norm(desc, None, None, None, None)
        dgamma, dbeta = torch.full((2, channels), 5.0, device="cuda")
        ws = torch.empty(wn.wino_layer_norm_backward_workspace_bytes(desc), dtype=torch.uint8, device="cuda")
        wn.wino_layer_norm_backward(desc, None, None, None, None, None, torch.empty(1, device="cuda"), dgamma, dbeta, ws)
        assert not dgamma.any() and not dbeta.any()


def test_rows_past_32_bit_offsets():
    """The last rows of a tensor of 2^32 elements and more, without touching the ones before."""
    import torch
    import paper_2004_11077_amd as wn
    rows, channels, stride = 70000, 64, 65536            # 4.6e9 elements of bf16: 9.2 GB
    whole = torch.empty(rows * stride, dtype=torch.bfloat16, device="cuda")
    x = whole.view(rows, stride)[:, :channels]
    x.copy_(torch.randn(rows, channels, device="cuda"))
    dense = x.contiguous()
    y, z = torch.empty(2, rows, channels, device="cuda")
    wn.wino_layer_norm(wn.NormDesc(rows, channels, x_type=wn.TYPE_BF16, x_stride=stride), x, None, None, y)
    wn.wino_layer_norm(wn.NormDesc(rows, channels, x_type=wn.TYPE_BF16), dense, None, None, z)
    assert torch.equal(y, z)
