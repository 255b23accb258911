"""int8 codes on the border between two: rint(y / s_y) of the formula, ties to even.  y is exactly beta where a row
has one value or gamma is zero, and (k + 1/2) s_y is exact in fp32 for s_y = n 2^-14 with few bits, so the
quotient is a tie and nothing but the formula's own rounding decides."""
import numpy as np
import pytest

from oracle import training as tr

pytestmark = pytest.mark.gpu

STEPS = [n * 2.0 ** -14 for n in (1, 3, 49, 99, 343, 1023, 1999)]


def codes(x, gamma, beta, s_y, stride=0):
    import torch
    import paper_2004_11077_amd as wn
    rows, channels = x.shape
    cuda = lambda a: None if a is None else torch.from_numpy(np.asarray(a, np.float32)).cuda()
    q = torch.full((rows, channels), 99, dtype=torch.int8, device="cuda")
    t = cuda(x)
    type = wn.TYPE_F32
    if (t.to(torch.bfloat16).float() == t).all():
        t, type = t.to(torch.bfloat16), wn.TYPE_BF16
    wn.wino_layer_norm(wn.NormDesc(rows, channels, x_type=type, y_type=wn.TYPE_I8, s_y=s_y), t, cuda(gamma), cuda(beta), q)
    return q.cpu().numpy()


def borders(channels, s_y):
    """(k + 1/2) s_y for all codes k, and two codes beyond them."""
    k = np.resize(np.arange(-130, 130), channels)
    return ((k + 0.5) * s_y).astype(np.float32)


@pytest.mark.parametrize("s_y", STEPS)
@pytest.mark.parametrize("channels", [255, 256, 20001])
def test_channels_without_a_weight(channels, s_y):
    rng = np.random.default_rng(channels)
    beta = borders(channels, s_y)
    got = codes(rng.standard_normal((5, channels)), np.zeros(channels), beta, s_y)
    assert np.array_equal(got, np.broadcast_to(tr.codes(beta.astype(np.float64), s_y), got.shape))


@pytest.mark.parametrize("channels", [96, 97, 20001])
@pytest.mark.parametrize("s_y", [2.0 ** -149, 1e-30, 0.03, 3e38])
def test_quotients_beyond_the_codes(channels, s_y):
    """Infinities and the largest values stop at the last code, NaN gives 0."""
    s_y = float(np.float32(s_y))
    beta = np.resize(np.float32([np.inf, -np.inf, 3.4e38, -3.4e38, 1e-45, -1e-45, 0, np.nan, 1, -300]), channels)
    with np.errstate(over="ignore", invalid="ignore"):
        want = np.clip(np.rint(beta.astype(np.float64) / s_y), -127, 127)
    got = codes(np.full((2, channels), 5.0), None, beta, s_y)
    assert np.array_equal(got, np.broadcast_to(np.nan_to_num(want).astype(np.int8), got.shape))


@pytest.mark.parametrize("s_y", STEPS)
@pytest.mark.parametrize("channels", [49, 63, 255, 256, 520, 2049, 20001])
def test_rows_of_one_value(channels, s_y):
    beta = borders(channels, s_y)
    assert (np.abs(beta.astype(np.float64) / s_y % 1) == 0.5).all()
    for values in ([3.25, -1000.0, 0.0, 2.0 ** 60], [1 / 3, 1e5 + 0.1, -7e-5, 1e20]):     # exact in bf16; in fp32 alone
        x = np.repeat(np.float32(values)[:, None], channels, 1)
        got = codes(x, None, beta, s_y)
        assert np.array_equal(got, np.broadcast_to(tr.codes(beta.astype(np.float64), s_y), got.shape)), values


@pytest.mark.parametrize("channels", [49, 70, 96, 2047, 3001, 20000])
def test_fp32_rows_of_one_value_are_beta(channels):
    """The sum of a row is exact here, and so is the mean: nothing is left beside it."""
    import torch
    import paper_2004_11077_amd as wn
    x = torch.tensor([1000.0, -3.0, 0.0, 96.5], device="cuda")[:, None].repeat(1, channels)
    beta = torch.randn(channels, device="cuda")
    y, mean = torch.empty_like(x), torch.empty(4, device="cuda")
    wn.wino_layer_norm(wn.NormDesc(4, channels), x, None, beta, y, mean)
    assert torch.equal(mean, x[:, 0]) and torch.equal(y, beta.expand_as(y))


@pytest.mark.parametrize("y_type", ["f32", "i8"])
@pytest.mark.parametrize("channels", [64, 100, 3001, 20001])
def test_rows_of_one_value_without_eps(channels, y_type):
    """rstd is 1 / sqrt(0), infinity, whatever comes out; y is 0 times that, NaN, whose code is 0."""
    import torch
    import paper_2004_11077_amd as wn
    x = torch.randn(4, channels, device="cuda")
    x[1], x[2] = 2.5, 0
    codes = y_type == "i8"
    y = torch.full((4, channels), 9, device="cuda").to(torch.int8 if codes else torch.float32)
    mean, rstd = torch.empty(2, 4, device="cuda")
    wn.wino_layer_norm(wn.NormDesc(4, channels, y_type=wn.TYPE_I8 if codes else wn.TYPE_F32, s_y=0.02, eps=0), x, None, None, y, mean, rstd)
    assert torch.isposinf(rstd[1:3]).all() and torch.isfinite(rstd[[0, 3]]).all()
    assert mean[1] == 2.5 and mean[2] == 0
    assert not y[1:3].any() if codes else torch.isnan(y[1:3]).all()
    ref, _, rrstd = tr.layer_norm(x[[0, 3]].double().cpu().numpy(), 1.0, 0.0, 0.0)
    if codes:
        assert np.array_equal(y[[0, 3]].cpu().numpy(), tr.codes(ref, 0.02))
