"""The binding of the training operators refuses tensors whose elements do not lie where a kernel looks for
them: expanded ones, whose memory is shorter than their shape, transposed and sliced ones.  Nothing is launched:
tensors of the CPU stand for the current device's, and every call is refused before the library sees it."""
import os

import pytest

torch = pytest.importorskip("torch")
wn = pytest.importorskip("paper_2004_11077_amd")
from paper_2004_11077_amd import binding  # noqa: E402

pytestmark = pytest.mark.skipif(not os.path.exists(wn.lib_path()),
                                reason="libwino.so not built (python -m paper_2004_11077_amd.build)")

R, C, V = 6, 8, 5


@pytest.fixture(autouse=True)
def tensors_of_the_cpu(monkeypatch):
    monkeypatch.setattr(binding, "_types", (lambda: -1, {wn.TYPE_F32: torch.float32, wn.TYPE_BF16: torch.bfloat16,
                                                         wn.TYPE_I8: torch.int8, "i64": torch.int64}))

    def no_call():
        raise AssertionError("a call that should have been refused reached the library")
    monkeypatch.setattr(binding, "_load", no_call)


def f(*shape, dtype=torch.float32):
    return torch.zeros(*shape, dtype=dtype)


def norm(**kw):
    a = dict(x=f(R, C), gamma=f(C), beta=f(C), y=f(R, C), mean=f(R), rstd=f(R)) | kw
    d = a.pop("desc", wn.NormDesc(R, C))
    wn.wino_layer_norm(d, *a.values(), stream=0)


def norm_backward(**kw):
    a = dict(dy=f(R, C), x=f(R, C), gamma=f(C), mean=f(R), rstd=f(R), dx=f(R, C), dgamma=f(C), dbeta=f(C), workspace=f(4096)) | kw
    d = a.pop("desc", wn.NormDesc(R, C))
    wn.wino_layer_norm_backward(d, *a.values(), stream=0)


def loss(**kw):
    a = dict(h=f(R, C), w=f(V, C), bias=f(V), targets=f(R, dtype=torch.int64), loss=f(R), lse=f(R), workspace=f(4096)) | kw
    d = a.pop("desc", wn.LossDesc(R, C, V))
    wn.wino_linear_cross_entropy(d, *a.values(), stream=0)


def loss_backward(**kw):
    a = dict(h=f(R, C), w=f(V, C), bias=f(V), targets=f(R, dtype=torch.int64), lse=f(R), dloss=f(R), dh=f(R, C), dw=f(V, C), dbias=f(V),
             workspace=f(4096)) | kw
    d = a.pop("desc", wn.LossDesc(R, C, V))
    wn.wino_linear_cross_entropy_backward(d, *a.values(), stream=0)


def update(**kw):
    a = dict(g=f(2, R, C), o=f(2, R, C), workspace=f(4096)) | kw
    d = a.pop("desc", wn.OrthogonaliseDesc(2, R, C))
    wn.wino_orthogonalise(d, *a.values(), stream=0)


ONE_RUN = {norm: ("x", "gamma", "beta", "y", "mean", "rstd"),
           norm_backward: ("dy", "x", "gamma", "mean", "rstd", "dx", "dgamma", "dbeta", "workspace"),
           loss: ("h", "w", "bias", "targets", "loss", "lse", "workspace"),
           loss_backward: ("h", "w", "bias", "targets", "lse", "dloss", "dh", "dw", "dbias", "workspace"),
           update: ("g", "o", "workspace")}
CASES = [(call, name) for call, names in ONE_RUN.items() for name in names]


def shape_and_type(name):
    """Of the argument that the call makes for itself."""
    rows = V if name in ("w", "dw") else R
    dtype = torch.int64 if name == "targets" else torch.float32
    if name in ("x", "y", "dy", "dx", "h", "w", "dh", "dw"):
        return (rows, C), dtype
    if name in ("g", "o"):
        return (2, R, C), dtype
    if name == "workspace":
        return (4096,), dtype
    return (V if name in ("bias", "dbias") else C if name in ("gamma", "beta", "dgamma", "dbeta") else R,), dtype


def refused(call, name, t, **kw):
    with pytest.raises(wn.WinoError) as e:
        call(**{name: t}, **kw)
    assert e.value.code == -1 and " %s " % name in " " + str(e.value).replace(":", " ") + " ", str(e.value)


@pytest.mark.parametrize("call,name", CASES, ids=lambda v: getattr(v, "__name__", v))
def test_one_element_seen_as_many(call, name):
    shape, dtype = shape_and_type(name)
    refused(call, name, torch.zeros((), dtype=dtype).expand(*shape))


@pytest.mark.parametrize("call,name", CASES, ids=lambda v: getattr(v, "__name__", v))
def test_slices_and_transposes_without_a_stride(call, name):
    shape, dtype = shape_and_type(name)
    refused(call, name, torch.zeros(*shape[:-1], 2 * shape[-1], dtype=dtype)[..., ::2])
    if len(shape) > 1:
        refused(call, name, torch.zeros(*shape[:-1], shape[-1] + 3, dtype=dtype)[..., :shape[-1]])
        refused(call, name, torch.zeros(*shape[:-2], shape[-1], shape[-2], dtype=dtype).transpose(-1, -2))


def test_a_gradient_of_a_mean():
    """What autograd hands on at the losses."""
    losses = torch.ones(R, requires_grad=True)
    got = []
    losses.register_hook(got.append)
    losses.sum().backward()
    assert got[0].stride() == (0,)
    refused(loss_backward, "dloss", got[0])


@pytest.mark.parametrize("bad", [
    torch.zeros(R, 12)[:, :C],                              # rows 12 apart, the descriptor says 10
    torch.zeros(R, 20)[:, :2 * C:2],                        # every other value
    torch.zeros(1, C).expand(R, C),                         # one row seen as many
    torch.zeros(C, R).t(),
    torch.zeros(200)[:R * C].view(R, C),                    # dense, though memory goes on behind it
    torch.as_strided(torch.zeros(200), (2, 3, C), (40, 10, 1)),   # rows 10 apart, but for the fourth
])
def test_rows_that_are_not_a_stride_apart(bad):
    for call, desc, names in ((norm, wn.NormDesc(R, C, x_stride=10, y_stride=10), ("x", "y")),
                              (norm_backward, wn.NormDesc(R, C, x_stride=10, dy_stride=10, dx_stride=10), ("x", "dy", "dx")),
                              (loss, wn.LossDesc(R, C, V, h_stride=10), ("h",)),
                              (loss_backward, wn.LossDesc(R, C, V, h_stride=10), ("h",))):
        good = {n: torch.zeros(R, 10)[:, :C] for n in names}
        for name in names:
            refused(call, name, bad, desc=desc, **{n: t for n, t in good.items() if n != name})


def test_matrices_that_are_not_a_stride_apart():
    d = wn.OrthogonaliseDesc(2, R, C, g_stride=10, g_batch=70)
    for bad in (torch.zeros(2, 7, 10)[:, :R, :C].transpose(0, 1), torch.as_strided(torch.zeros(200), (2, R, C), (71, 10, 1)),
                torch.as_strided(torch.zeros(200), (2, R, C), (0, 10, 1)), torch.as_strided(torch.zeros(200), (2, R, C), (70, 9, 1))):
        refused(update, "g", bad, desc=d)


def test_tensors_that_lie_as_they_should():
    F = wn.TYPE_F32
    x = torch.zeros(3, 4, 5, 10)
    binding._fit(("gamma", f(C), F, C), ("longer", f(C + 3), F, C), ("shaped", f(2, 4), F, C), ("none", None, F, C),
                 ("slice", f(20)[3:11], F, C), ("one", f(9)[::9], F, 1), ("room", f(0), None, 0))
    binding._fit_rows(
        ("dense", f(R, C), F, 0, R, C), ("the same", f(R, C), F, C, R, C), ("pixels", x, F, 0, 60, 10), ("filters", f(4, 3, 3, 3), F, 0, 4, 27),
        ("part of the channels", x[..., 2:9], F, 10, 60, 7), ("more rows", x[..., :7], F, 10, 31, 7), ("one row", x[0, 0, :1, :7], F, 999, 1, 7),
        ("one value", x[..., 0], F, 10, 60, 1), ("of many rows", f(5, 9)[:, :4], F, 9, 1, 4), ("no rows", x.expand(2, 3, 4, 5, 10), F, 0, 0, 7),
        ("one run", f(100), F, 11, 9, 7), ("batch", torch.as_strided(f(300), (2, R, C), (70, 10, 1), 5), F, 10, R, C, 70, 2),
        ("dense matrices apart", torch.as_strided(f(300), (2, R, C), (70, C, 1)), F, 0, R, C, 70, 2),
        ("rows apart, matrices on", f(2, R, 10)[..., :C], F, 10, R, C, 0, 2), ("filters apart", f(2, 4, 30)[..., :27].unflatten(2, (3, 3, 3)), F, 30, 4, 27, 0, 2))
    for bad in (("short", f(C - 1), F, C), ("type", f(C, dtype=torch.bfloat16), F, C)):
        with pytest.raises(wn.WinoError):
            binding._fit(bad)


def test_channels_last_in_memory():
    """[N][C][H][W] with the channels last in memory is [N][H][W][C]."""
    F, last = wn.TYPE_F32, torch.channels_last
    x = torch.zeros(2, 7, 3, 4).to(memory_format=last)
    assert not x.is_contiguous()
    binding._fit_rows(("dense", x, F, 0, 24, 7), ("some of them", torch.zeros(2, 10, 3, 4).to(memory_format=last)[:, :7], F, 10, 24, 7))
    for bad in (("rows of others", x, F, 0, 42, 4), ("apart", x, F, 10, 24, 7), ("first", torch.zeros(2, 4, 7, 3).permute(0, 2, 3, 1), F, 0, 24, 7),
                ("some", torch.zeros(2, 10, 3, 4).to(memory_format=last)[:, :7], F, 0, 24, 7)):
        with pytest.raises(wn.WinoError):
            binding._fit_rows(bad)


def test_filters_with_channels_last_in_memory(monkeypatch):
    """One order of the columns in both is as good as another; in one of them alone it is not."""
    class Library:
        def __getattr__(self, name):
            return lambda *args: 0
    d = wn.OrthogonaliseDesc(1, R, 9 * C)
    last = f(R, C, 3, 3).to(memory_format=torch.channels_last)
    refused(update, "g", last, o=f(R, C, 3, 3), desc=d)
    refused(update, "o", last, g=f(R, C, 3, 3), desc=d)
    refused(update, "g", f(C, R, 3, 3).transpose(0, 1), o=f(C, R, 3, 3).transpose(0, 1), desc=d)
    monkeypatch.setattr(binding, "_load", Library)
    update(g=last, o=torch.empty_like(last), desc=d)
    update(g=f(R, C, 3, 3), o=f(R, C, 3, 3), desc=d)
