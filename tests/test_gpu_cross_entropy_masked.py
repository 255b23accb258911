"""Classes that a bias of -infinity masks count for nothing, whatever finite values their weights hold: the weights of a
padded vocabulary's last classes may never have been set."""
import numpy as np
import pytest

from test_gpu_cross_entropy import check, run

pytestmark = pytest.mark.gpu

# planes, in one piece and several, fp32 as it stands, bf16
SHAPES = [(40, 64, 300, "f32", 0), (300, 128, 700, "f32", 256), (1001, 67, 1030, "f32", 0), (700, 520, 1025, "f32", 512),
          (40, 130, 1031, "f32", 0), (2000, 67, 5, "f32", 0), (300, 128, 700, "bf16", 0), (40, 130, 300, "bf16", 0)]


@pytest.mark.parametrize("value", [1e30, 3e38, -1e25])
@pytest.mark.parametrize("T,D,V,type,piece", SHAPES)
def test_weights_of_masked_classes(T, D, V, type, piece, value):
    """Bit for bit what zeros give."""
    masked = np.r_[0:V // 3, V - 1]

    def change(v):
        def f(h, w, b, target, dloss):
            b[masked] = -np.inf
            target[np.isin(target, masked)] = V // 2
            h.mul_(1e-3)                      # no product of an h and a masked w overflows
            for i in masked:
                w[int(i)] = v
        return f
    got, zero = (run(T, D, V, type, piece=piece, change=change(v), extra=int(T == 40)) for v in (value, 0))
    for name in ("loss", "lse", "dh", "dw", "dbias"):
        assert np.array_equal(got[name], zero[name]), name
    assert not got["dw"][masked].any() and not got["dbias"][masked].any()
    check(zero, type)


@pytest.mark.parametrize("T,D,V,type,piece", SHAPES)
def test_masked_targets(T, D, V, type, piece):
    """A masked class that is a row's target has a gradient: its weights count, also where they are larger than
    all others."""
    def change(h, w, b, target, dloss):
        b[::2] = -np.inf
        w[::2].mul_(1000)
        h.mul_(1e-3)
        target[:] = np.where(target % 4 == 2, target, target | 1) % V
    r = run(T, D, V, type, piece=piece, change=change)
    k = (r["target"] >= 0) & (r["target"] < V)
    assert np.isposinf(r["loss"][k & (r["target"] % 2 == 0)]).all() and (k & (r["target"] % 2 == 0)).any()
    check(r, type)


@pytest.mark.parametrize("T,D,V,type,piece", SHAPES)
def test_products_that_overflow(T, D, V, type, piece):
    """A masked class's logit is -infinity also where h times its weights is +infinity."""
    masked = np.r_[0:V // 3, V - 1]

    def change(v):
        def f(h, w, b, target, dloss):
            b[masked] = -np.inf
            target[np.isin(target, masked)] = V // 2
            h.abs_()
            for i in masked:
                w[int(i)] = v
        return f
    got, zero = (run(T, D, V, type, piece=piece, change=change(v)) for v in (3.3e38, 0))
    for name in ("loss", "lse", "dh", "dw", "dbias"):
        assert np.array_equal(got[name], zero[name]), name
    check(zero, type)
