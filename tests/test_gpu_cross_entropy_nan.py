"""Loss gradients that are no numbers: the formula multiplies by them, so what they touch is NaN, and nothing
else is.  A program that looks for NaN in its gradients, as one that scales its losses does, finds it."""
import numpy as np
import pytest

from test_gpu_cross_entropy import check, run

pytestmark = pytest.mark.gpu

# planes, fp32 as it stands (2^16 weights, or few classes of 2^16 features), bf16 in tiles of 32 and 64
SHAPES = [(1, 64, 30, "f32"), (40, 64, 300, "f32"), (1, 130, 1031, "f32"), (40, 130, 1031, "f32"), (2000, 67, 3, "f32"),
          (300, 128, 700, "f32"), (1, 64, 30, "bf16"), (40, 130, 300, "bf16"), (300, 128, 700, "bf16")]


@pytest.mark.parametrize("T,D,V,type", SHAPES)
@pytest.mark.parametrize("others", ["nan", "zero"])
def test_no_row_has_a_number(T, D, V, type, others):
    """All NaN, as behind the mean of a NaN loss, or one NaN and zeros."""
    def change(h, w, b, target, dloss):
        dloss[:] = np.nan if others == "nan" else 0
        dloss[T // 2] = np.nan
        target[T // 2] = V // 2
    r = run(T, D, V, type, ignored=0.1, change=change)
    k = (r["target"] >= 0) & (r["target"] < V)
    gone = k & np.isnan(r["dloss"])
    assert np.isnan(r["dh"][gone]).all() and not r["dh"][~gone].any()
    assert np.isnan(r["dw"]).all() and np.isnan(r["dbias"]).all()


@pytest.mark.parametrize("value", [np.nan, np.inf, -np.inf])
@pytest.mark.parametrize("T,D,V,type", [s for s in SHAPES if s[0] > 1])
def test_beside_rows_that_have_one(T, D, V, type, value):
    """The other rows' dh is what it is when the row's dloss is zero, bit for bit."""
    at = T // 3

    def change(v):
        def f(h, w, b, target, dloss):
            target[at], dloss[at] = 1, v
        return f
    r, zero = (run(T, D, V, type, change=change(v)) for v in (value, 0))
    rest = np.arange(T) != at
    assert np.array_equal(r["dh"][rest], zero["dh"][rest])
    assert not np.isfinite(r["dh"][at]).any() and not np.isfinite(r["dw"]).any() and not np.isfinite(r["dbias"]).any()
    assert np.array_equal(r["loss"], zero["loss"])
    check(zero, type)


def test_every_class_masked_has_no_gradient():
    """Whatever dloss is."""
    def change(h, w, b, target, dloss):
        b[:], dloss[::2] = -np.inf, np.nan
    for type in ("f32", "bf16"):
        r = run(30, 64, 200, type, ignored=0, change=change)
        assert not r["dh"].any() and not r["dw"].any() and not r["dbias"].any()
